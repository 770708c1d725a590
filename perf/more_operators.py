"""Cases and plain forms of the operators of sparse language models and their teachers: routing of tokens to
experts, products grouped by expert, the experts' results combined, distillation from a teacher's top logits.

Workers come first, as in the library's state: every worker has its own router and experts.  `run` computes an
operator in elementary torch operations (own = False) or calls the library (own = True).
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------ cases

def listed():
    return [
        # the next token of eight sequences, eight of 64 experts each
        dict(name="route decode", op="route", m=1, T=8, E=64, k=8, normalise=True, dtype="fp32", train=False),
        # a training batch through many small experts; padding at the sequences' ends goes nowhere
        dict(name="route train", op="route", m=2, T=16384, E=128, k=8, normalise=False, dtype="fp32", train=True),
        # the experts' answers for eight tokens
        dict(name="combine decode", op="combine", m=1, T=8, k=8, D=1024, dtype="bf16", train=False),
        # a training batch, two experts a token
        dict(name="combine train", op="combine", m=1, T=16384, k=2, D=1024, dtype="bf16", train=True),
        # 16 workers of odd width: no row but the first starts on a 16-byte boundary
        dict(name="combine odd", op="combine", m=16, T=333, k=3, D=1021, dtype="fp16", train=True),
        # sixteen rows spread over 64 experts: only weights count
        dict(name="product decode", op="product", m=1, R=16, E=64, D=1024, F=2048, dtype="bf16", train=False),
        # the worker-stacked training step: 16 workers with four experts each
        dict(name="product 16 workers", op="product", m=16, R=512, E=4, D=1024, F=1024, dtype="bf16", train=True),
        # odd widths, ragged groups, experts that no token chose
        dict(name="product odd", op="product", m=3, R=1001, E=11, D=1021, F=515, dtype="fp16", train=True),
        # a long batch through eight wide experts, two for each token
        dict(name="product large", op="product", m=1, R=32768, E=8, D=2048, F=4096, dtype="bf16", train=True),
        # ten-class heads of 16 workers with batch 128, taught by another model's three best classes
        dict(name="distill ten classes", op="distill", N=2048, V=10, K=3, temperature=2.0, dtype="fp32", train=True, masked=False),
        # a training step's loss over a vocabulary: the teacher's 32 best tokens, kept on disk
        dict(name="distill train", op="distill", N=4096, V=32768, K=32, temperature=1.0, dtype="bf16", train=True, masked=False),
        # evaluation against a teacher: odd vocabulary, part of it masked out with -inf
        dict(name="distill odd", op="distill", N=1021, V=50021, K=20, temperature=1.5, dtype="fp32", train=False, masked=True),
    ]


def _log_between(rng, low, high):
    return int(min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["route", "combine", "product", "product", "distill", "distill"])
    if op == "route":
        c = dict(op=op, m=rng.choice([1, 1, 2, 4]), T=_log_between(rng, 1, 8192), E=_log_between(rng, 2, 256),
                 normalise=rng.random() < 0.5, dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]), train=rng.random() < 0.6)
        c["k"] = min(c["E"], rng.choice([1, 2, 2, 4, 6, 8]))
        return c
    if op == "combine":
        while True:
            c = dict(op=op, m=rng.choice([1, 1, 2, 4, 16]), T=_log_between(rng, 1, 16384), k=rng.choice([1, 2, 2, 3, 4, 6, 8]),
                     D=_log_between(rng, 16, 4096), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), train=rng.random() < 0.6)
            if rng.random() < 0.5:
                c["D"] = max(16, c["D"] // 16 * 16)
            if c["m"] * c["T"] * c["k"] * c["D"] <= 16384 * 2 * 1024:
                return c
    if op == "product":
        while True:
            c = dict(op=op, m=rng.choice([1, 1, 1, 2, 4, 16]), R=_log_between(rng, 1, 32768), E=_log_between(rng, 1, 128),
                     D=_log_between(rng, 32, 4096), F=_log_between(rng, 32, 4096), dtype=rng.choice(["bf16", "fp16"]), train=rng.random() < 0.6)
            if rng.random() < 0.6:  # widths of whole 16-byte pieces, as models have them
                c["D"], c["F"] = max(32, c["D"] // 32 * 32), max(32, c["F"] // 32 * 32)
            if (c["m"] * c["R"] * c["D"] * c["F"] <= 32768 * 2048 * 4096 and c["m"] * c["E"] * c["D"] * c["F"] <= 1 << 27
                    and c["m"] * c["R"] * max(c["D"], c["F"]) <= 1 << 27):
                return c
    while True:
        c = dict(op="distill", N=_log_between(rng, 1, 8192), V=_log_between(rng, 2, 200000), temperature=rng.choice([1.0, 1.0, 1.5, 2.0, 4.0]),
                 dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), train=rng.random() < 0.6, masked=rng.random() < 0.3)
        c["K"] = min(c["V"], rng.choice([1, 4, 8, 20, 32, 64, 128]))
        if c["V"] < 512:
            c["masked"] = False
        if c["N"] * c["V"] <= 4096 * 32768:
            return c


# ----------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _group_sizes(c, seed):
    """Rows of each worker's experts: some experts are several times as popular as others; one row in fifty is padding, behind
    the last expert's."""
    rng = random.Random(seed)
    out = []
    for _ in range(c["m"]):
        weights = [math.exp(rng.gauss(0.0, 0.7)) for _ in range(c["E"])]
        live = c["R"] - c["R"] // 50
        if live <= 4096:
            n = [0] * c["E"]
            for e in rng.choices(range(c["E"]), weights, k=live):
                n[e] += 1
        else:
            total, n = sum(weights), []
            for w in weights:
                n.append(min(live - sum(n), int(live * w / total + rng.random())))
            n[0] += live - sum(n)
        out.append(n)
    return out


def prepare(case, seed):
    c, g = case, _generator(seed)
    dtype = _TYPES[c["dtype"]]
    s = dict(case)
    if c["op"] == "route":
        m, T, E, k = c["m"], c["T"], c["E"], c["k"]
        s["logits"] = _normal(g, (m, T, E), dtype, 1.5)
        if T > 16:  # padding
            s["logits"].masked_fill_(torch.rand((m, T, 1), generator=g, device="cuda") < 0.03, -math.inf)
        if c["train"]:
            s["dw"] = _normal(g, (m, T, k), torch.float32)
    elif c["op"] == "combine":
        m, T, k, D = c["m"], c["T"], c["k"], c["D"]
        R = T * k
        s["rows"] = _normal(g, (m, R, D), dtype)
        # any order of the slots, as experts leave it; padded tokens have no rows, and leave as many behind the others
        order = torch.stack([torch.randperm(R, generator=g, device="cuda") for _ in range(m)])
        gone = torch.rand((m, T), generator=g, device="cuda") < (0.03 if T > 16 else -1.0)
        live = ~gone.repeat_interleave(k, dim=1).gather(1, order)
        order = order.gather(1, torch.sort((~live).to(torch.int8), dim=1, stable=True).indices)
        n = live.sum(dim=1, keepdim=True)
        rank = torch.arange(R, device="cuda")[None].expand(m, R)
        s["tokens"] = torch.where(rank < n, order // k, -1).to(torch.int32)
        places = torch.empty((m, R), dtype=torch.int64, device="cuda").scatter_(1, order, torch.where(rank < n, rank, -1))
        s["places"] = places.to(torch.int32).view(m, T, k)
        w = torch.softmax(_normal(g, (m, T, k), torch.float32), dim=-1)
        s["weights"] = torch.where(s["places"] < 0, 0.0, w)
        if c["train"]:
            s["dy"] = _normal(g, (m, T, D), dtype)
    elif c["op"] == "product":
        m, R, E, D, F = c["m"], c["R"], c["E"], c["D"], c["F"]
        s["sizes"] = _group_sizes(c, seed)
        s["offsets"] = torch.tensor([[sum(n[:e]) for e in range(E + 1)] for n in s["sizes"]], dtype=torch.int32, device="cuda")
        s["x"] = _normal(g, (m, R, D), dtype)
        s["w"] = _normal(g, (m, E, F, D), dtype, D ** -0.5)
        if c["train"]:
            s["dy"] = _normal(g, (m, R, F), dtype)
    else:
        N, V, K = c["N"], c["V"], c["K"]
        s["logits"] = _normal(g, (N, V), dtype, 3.0)
        if c["masked"]:
            s["logits"].masked_fill_(torch.rand((N, V), generator=g, device="cuda") < 0.25, -math.inf)
        # distinct tokens: a random start and a stride of its own for each row
        start = torch.randint(0, V, (N, 1), generator=g, device="cuda")
        ids = (start + torch.arange(K, device="cuda") * max(1, V // K)) % V
        # the teacher mostly likes what the student likes, too
        s["logits"].scatter_(1, ids, _normal(g, (N, K), dtype, 3.0))
        s["teacher"] = torch.sort(_normal(g, (N, K), dtype, 3.0).float(), dim=1, descending=True).values.to(dtype)
        # positions of padding have no teacher
        s["ids"] = torch.where(torch.rand((N, 1), generator=g, device="cuda") < 0.03, -1, ids).to(torch.int32)
        if c["train"]:
            s["dloss"] = torch.rand((N,), generator=g, device="cuda") / N
    return s


# -------------------------------------------------------------------------- one pass

def run(state):
    s = state
    if own:
        import paper_2002_09539_b200 as lib
        if s["op"] == "route":
            r = lib.expert_route(s["logits"], s["k"], s["normalise"])
            out = {"weights": r.weights, "ids": r.ids, "places": r.places, "tokens": r.tokens, "offsets": r.offsets}
            if s["train"]:
                out["dlogits"] = lib.expert_route_backward(s["dw"], s["logits"], r.ids, r.weights, s["normalise"])
            return out
        if s["op"] == "combine":
            out = {"y": lib.expert_combine(s["rows"], s["places"], s["weights"])}
            if s["train"]:
                out["drows"], out["dweights"] = lib.expert_combine_backward(s["dy"], s["rows"], s["places"], s["tokens"], s["weights"])
            return out
        if s["op"] == "product":
            out = {"y": lib.expert_product(s["x"], s["w"], s["offsets"])}
            if s["train"]:
                out["dx"], out["dw"] = lib.expert_product_backward(s["dy"], s["x"], s["w"], s["offsets"])
            return out
        # the weight of a row's loss is known ahead, so its gradient comes with it
        r = lib.distill_loss(s["logits"], s["ids"], s["teacher"], s["temperature"], d_loss=s["dloss"] if s["train"] else None)
        return {"loss": r.loss, "dlogits": r.d_logits} if s["train"] else {"loss": r.loss}
    return {"route": _route, "combine": _combine, "product": _product, "distill": _distill}[s["op"]](s)


def _route(s):
    x, k = s["logits"].float(), s["k"]
    m, T, E = x.shape
    v, i = torch.sort(x, dim=2, descending=True, stable=True)
    v, i = v[..., :k], i[..., :k]
    none = v == -math.inf
    top = torch.where(none[..., :1], 0.0, v[..., :1])
    e = torch.exp(v - top)
    total = e.sum(dim=2, keepdim=True) if s["normalise"] else torch.exp(x - top).sum(dim=2, keepdim=True)
    w = torch.where(none, 0.0, e / total)
    ids = torch.where(none, E, i)
    # rows by expert, tokens in order within one; what goes nowhere comes last
    flat = ids.reshape(m, T * k)
    order = torch.sort(flat, dim=1, stable=True).indices
    counts = torch.zeros((m, E + 1), dtype=torch.int64, device=x.device).scatter_add_(1, flat, torch.ones_like(flat))
    offsets = torch.cumsum(counts, dim=1) - counts
    rank = torch.arange(T * k, device=x.device)[None].expand(m, T * k)
    there = rank < offsets[:, E:]
    places = torch.empty_like(flat).scatter_(1, order, torch.where(there, rank, -1))
    out = {"weights": w, "ids": torch.where(none, -1, i).to(torch.int32), "places": places.to(torch.int32).view(m, T, k),
           "tokens": torch.where(there, order // k, -1).to(torch.int32), "offsets": offsets.to(torch.int32)}
    if s["train"]:
        dw = torch.where(none, 0.0, s["dw"])
        mean = (w * dw).sum(dim=2, keepdim=True)
        if s["normalise"]:
            d = torch.zeros_like(x).scatter_(2, i, torch.where(none, 0.0, w * (dw - mean)))
        else:
            p = torch.where(none[..., :1], 0.0, torch.exp(x - top) / total)
            d = p * (torch.zeros_like(x).scatter_(2, i, dw) - mean)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _combine(s):
    rows, places, w = s["rows"].float(), s["places"].long(), s["weights"]
    m, T, k = places.shape
    worker = torch.arange(m, device=rows.device)[:, None]
    there = (places >= 0)[..., None]
    y = torch.zeros((m, T, rows.shape[2]), device=rows.device)
    for j in range(k):
        y = y + torch.where(there[:, :, j], w[:, :, j, None] * rows[worker, places[:, :, j].clamp(min=0)], 0.0)
    out = {"y": y.to(s["rows"].dtype)}
    if s["train"]:
        dy, drows, dw = s["dy"].float(), torch.zeros_like(rows), torch.zeros_like(w)
        for j in range(k):
            at, has = places[:, :, j].clamp(min=0), there[:, :, j]
            dw[:, :, j] = torch.where(has[..., 0], (dy * rows[worker, at]).sum(dim=2), 0.0)
            # (adding zeros to row 0 where there is none)
            drows.index_put_((worker.expand(m, T), at), torch.where(has, w[:, :, j, None] * dy, 0.0), accumulate=True)
        out["drows"], out["dweights"] = drows.to(s["rows"].dtype), dw
    return out


def _product(s):
    x, w = s["x"].float(), s["w"].float()
    y = torch.zeros((x.shape[0], x.shape[1], w.shape[2]), device=x.device)
    if s["train"]:
        dy, dx, dw = s["dy"].float(), torch.zeros_like(x), torch.zeros_like(w)
    for i, sizes in enumerate(s["sizes"]):
        a = 0
        for e, n in enumerate(sizes):
            if n:
                y[i, a:a + n] = x[i, a:a + n] @ w[i, e].T
                if s["train"]:
                    dx[i, a:a + n] = dy[i, a:a + n] @ w[i, e]
                    dw[i, e] = dy[i, a:a + n].T @ x[i, a:a + n]
            a += n
    t = s["x"].dtype
    return {"y": y.to(t), "dx": dx.to(t), "dw": dw.to(t)} if s["train"] else {"y": y.to(t)}


def _distill(s):
    scale = 1.0 / s["temperature"]
    x, z, ids = s["logits"].float() * scale, s["teacher"].float() * scale, s["ids"].long()
    has = ids >= 0
    z = torch.where(has, z, -math.inf)
    top = z.amax(dim=1, keepdim=True)
    gone = top == -math.inf
    e = torch.exp(z - torch.where(gone, 0.0, top))
    q = torch.where(gone, 0.0, e / e.sum(dim=1, keepdim=True))
    logq = z - torch.where(gone, 0.0, top) - torch.log(e.sum(dim=1, keepdim=True))
    xt = x.amax(dim=1, keepdim=True)
    ex = torch.exp(x - xt)
    total = ex.sum(dim=1, keepdim=True)
    lp = x.gather(1, ids.clamp(min=0)) - xt - torch.log(total)
    out = {"loss": torch.where(q > 0, q * (logq - lp), 0.0).sum(dim=1)}
    if s["train"]:
        d = torch.where(gone, 0.0, ex / total).scatter_add_(1, ids.clamp(min=0), -q)
        out["dlogits"] = (d * (s["dloss"][:, None] * scale)).to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------ work

def work(case):
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "route":
        n, slots = c["m"] * c["T"] * c["E"], c["m"] * c["T"] * c["k"]
        # logits in; weights, ids, places and tokens out; training adds the weights' gradients in and the logits' out
        return {"bytes": n * e * (2 if c["train"] else 1) + slots * (20 if c["train"] else 16) + 4 * c["m"] * (c["E"] + 1),
                "flops": n * (5 if c["train"] else 2)}
    if c["op"] == "combine":
        n, slots = c["m"] * c["T"] * c["D"], c["m"] * c["T"] * c["k"]
        # rows in, tokens out; training adds the tokens' gradients in and the rows' out
        b = e * n * (c["k"] + 1) + 8 * slots
        f = 2 * n * c["k"]
        if c["train"]:
            b += e * n * (c["k"] + 1) + 8 * slots
            f += 3 * n * c["k"]
        return {"bytes": b, "flops": f}
    if c["op"] == "product":
        m, R, D, F = c["m"], c["R"], c["D"], c["F"]
        # no more experts are read than there are rows
        b = e * m * (R * D + min(c["E"], R) * F * D + R * F)
        f = 2 * m * R * D * F
        if c["train"]:
            b += e * m * (R * F + R * D + c["E"] * F * D)
            f += 4 * m * R * D * F
        return {"bytes": b, "flops": f}
    n = c["N"] * c["V"]
    return {"bytes": n * e * (2 if c["train"] else 1) + c["N"] * (c["K"] * (4 + e) + (8 if c["train"] else 4)),
            "flops": n * (6 if c["train"] else 3)}


# ----------------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    if s["op"] == "route":
        x, k = s["logits"].double(), s["k"]
        m, T, E = x.shape
        value, index = x.topk(k, dim=2)
        # (equal logits: the lowest expert first)
        key = x.float().contiguous()
        index = torch.argsort(-key, dim=2, stable=True)[..., :k]
        value = x.gather(2, index)
        live = torch.isfinite(value)
        lse = torch.logsumexp(value if s["normalise"] else x, dim=2, keepdim=True)
        w = torch.exp(value - lse).masked_fill(~live, 0.0)
        ids = index.masked_fill(~live, -1)
        places = torch.full((m, T * k), -1, dtype=torch.int64, device=x.device)
        tokens = torch.full((m, T * k), -1, dtype=torch.int64, device=x.device)
        offsets = torch.zeros((m, E + 1), dtype=torch.int64, device=x.device)
        for i in range(m):
            f = ids[i].reshape(-1)
            used = torch.nonzero(f >= 0)[:, 0]
            chosen = used[torch.argsort(f[used], stable=True)]
            places[i, chosen] = torch.arange(len(chosen), device=x.device)
            tokens[i, :len(chosen)] = torch.div(chosen, k, rounding_mode="floor")
            offsets[i, 1:] = torch.cumsum(torch.bincount(f[used], minlength=E), 0)
        out = {"weights": w, "ids": ids.to(torch.int32), "places": places.to(torch.int32).view(m, T, k), "tokens": tokens.to(torch.int32),
               "offsets": offsets.to(torch.int32)}
        if s["train"]:
            G = torch.zeros_like(x).scatter_add_(2, index, s["dw"].double() * live)
            chosen = torch.zeros_like(x).scatter_add_(2, index, live.double())
            p = torch.exp(x - lse).nan_to_num(0.0)
            if s["normalise"]:
                p = p * chosen
            out["dlogits"] = p * G - p * (p * G).sum(dim=2, keepdim=True)
        return out
    if s["op"] == "combine":
        m, T, k = s["places"].shape
        R, D = s["rows"].shape[1:]
        ys, drs, dws = [], [], []
        for i in range(m):
            P, W, X = s["places"][i].reshape(-1).long(), s["weights"][i].reshape(-1).double(), s["rows"][i].double()
            slot = torch.nonzero(P >= 0)[:, 0]
            token = torch.div(slot, k, rounding_mode="floor")
            ys.append(torch.zeros((T, D), dtype=torch.float64, device=X.device).index_add_(0, token, X[P[slot]] * W[slot, None]))
            if s["train"]:
                g = s["dy"][i].double()[token]
                dr, dw = torch.zeros_like(X), torch.zeros_like(W)
                dr[P[slot]] = g * W[slot, None]
                dw[slot] = torch.einsum("sd,sd->s", g, X[P[slot]])
                drs.append(dr)
                dws.append(dw.view(T, k))
        out = {"y": torch.stack(ys)}
        if s["train"]:
            out["drows"], out["dweights"] = torch.stack(drs), torch.stack(dws)
        return out
    if s["op"] == "product":
        ends = s["offsets"].tolist()
        m, R, D = s["x"].shape
        E, F = s["w"].shape[1:3]
        out = {"y": torch.zeros((m, R, F), dtype=torch.float64, device="cuda")}
        if s["train"]:
            out["dx"] = torch.zeros((m, R, D), dtype=torch.float64, device="cuda")
            out["dw"] = torch.zeros((m, E, F, D), dtype=torch.float64, device="cuda")
        for i in range(m):
            for e in range(E):
                part = slice(ends[i][e], ends[i][e + 1])
                X, W = s["x"][i, part].double(), s["w"][i, e].double()
                out["y"][i, part] = torch.einsum("rd,fd->rf", X, W)
                if s["train"]:
                    G = s["dy"][i, part].double()
                    out["dx"][i, part] = torch.einsum("rf,fd->rd", G, W)
                    out["dw"][i, e] = torch.einsum("rf,rd->fd", G, X)
        return out
    t = s["temperature"]
    live = s["ids"] >= 0
    at = s["ids"].long().clamp(min=0)
    lq = torch.log_softmax((s["teacher"].double() / t).masked_fill(~live, -1e300), dim=1)
    q = torch.exp(lq) * live
    lp = torch.log_softmax(s["logits"].double() / t, dim=1)
    out = {"loss": (torch.xlogy(q, q) - q * lp.gather(1, at).masked_fill(~live, 0.0)).sum(dim=1)}
    if s["train"]:
        d = torch.exp(lp) * live.any(dim=1, keepdim=True)
        d.scatter_add_(1, at, -q)
        out["dlogits"] = d * (s["dloss"].double() / t)[:, None]
    return out
