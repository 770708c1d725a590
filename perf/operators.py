"""Cases and plain forms of the operators on caller-owned tensors: gated feed-forward block, token log
probabilities, embedding lookup, per-worker gradient clipping.

All tensors carry the worker dimension first, as the library's state does.  `run` computes an
operator in elementary torch operations (own = False) or calls the library (own = True).
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------ cases

def listed():
    return [
        # serving one token: both projections are read once, nothing else matters
        dict(name="gated token", op="gated", m=1, T=1, D=1024, F=4096, act="silu", dtype="bf16", train=False),
        # the worker-stacked training step: 16 workers, batch 128, hidden widths of 1024
        dict(name="gated 16 workers", op="gated", m=16, T=128, D=1024, F=1024, act="relu", dtype="bf16", train=True),
        # odd widths and a ragged token count: no row starts on a 16-byte boundary
        dict(name="gated odd", op="gated", m=3, T=333, D=1021, F=2035, act="gelu", dtype="fp16", train=True),
        # a long batch through one wide block
        dict(name="gated large", op="gated", m=1, T=8192, D=4096, F=8192, act="silu", dtype="bf16", train=True),
        # the next token of eight sequences, with the twenty most likely alternatives
        dict(name="logprobs decode", op="logprobs", N=8, V=131072, top=20, dtype="bf16", train=False, masked=False),
        # ten-class heads of 16 workers with batch 128
        dict(name="logprobs ten classes", op="logprobs", N=2048, V=10, top=1, dtype="fp32", train=True, masked=False),
        # a training step's loss over a vocabulary
        dict(name="logprobs train", op="logprobs", N=4096, V=32768, top=0, dtype="bf16", train=True, masked=False),
        # scoring of given texts: odd vocabulary, part of it masked out with -inf
        dict(name="logprobs odd", op="logprobs", N=1021, V=50021, top=5, dtype="fp32", train=False, masked=True),
        # lookup for a prompt
        dict(name="embedding lookup", op="embedding", m=1, T=4096, V=32768, D=1024, dtype="bf16", train=False),
        # a training step's input layer: lookup, and the table's gradient in fp32
        dict(name="embedding train", op="embedding", m=2, T=16384, V=32768, D=1024, dtype="bf16", train=True),
        # the flat gradient rows that the local step takes
        dict(name="clip flat", op="clip", m=16, count=1, most=10000000, dtype="fp32", widen=False),
        # the gradients of a model's many layers, clipped and widened to fp32
        dict(name="clip many", op="clip", m=4, count=48, most=1000000, dtype="bf16", widen=True),
    ]


def _log_between(rng, low, high):
    return int(min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["gated", "gated", "logprobs", "logprobs", "embedding", "clip"])
    if op == "gated":
        while True:
            c = dict(op=op, m=rng.choice([1, 1, 2, 3, 4, 8, 16]), T=_log_between(rng, 1, 8192), D=_log_between(rng, 32, 4096),
                     F=_log_between(rng, 32, 8192), act=rng.choice(["silu", "gelu", "relu", "sigmoid"]),
                     dtype=rng.choice(["bf16", "fp16"]), train=rng.random() < 0.6)
            if rng.random() < 0.5:  # widths of whole 16-byte pieces, as models have them
                c["D"], c["F"] = max(32, c["D"] // 32 * 32), max(32, c["F"] // 32 * 32)
            if c["m"] * c["T"] * c["D"] * c["F"] <= 8192 * 4096 * 8192 and c["m"] * c["D"] * c["F"] <= 1 << 27 and c["m"] * c["T"] * c["F"] <= 1 << 26:
                return c
    if op == "logprobs":
        while True:
            c = dict(op=op, N=_log_between(rng, 1, 8192), V=_log_between(rng, 2, 200000), dtype=rng.choice(["bf16", "fp16", "fp32"]),
                     train=rng.random() < 0.5, masked=rng.random() < 0.3)
            c["top"] = min(c["V"], rng.choice([0, 1, 5, 20, 32]))
            if c["top"] > 0 and c["V"] < 64:
                c["masked"] = False
            if c["N"] * c["V"] <= 4096 * 32768 and (c["top"] == 0 or c["N"] * c["V"] <= 1021 * 50021):
                return c
    if op == "embedding":
        while True:
            c = dict(op=op, m=rng.choice([1, 1, 2, 4, 8]), T=_log_between(rng, 1, 32768), V=_log_between(rng, 10, 65536),
                     D=_log_between(rng, 8, 2048), dtype=rng.choice(["bf16", "fp16", "fp32"]), train=rng.random() < 0.7)
            if rng.random() < 0.5:
                c["D"] = max(8, c["D"] // 8 * 8)
            if c["m"] * c["V"] * c["D"] <= 2 * 32768 * 1024 and c["m"] * c["T"] * c["D"] <= 2 * 16384 * 1024:
                return c
    while True:
        c = dict(op=op, m=rng.choice([1, 2, 4, 8, 16]), count=_log_between(rng, 1, 48), most=_log_between(rng, 100, 10000000),
                 dtype=rng.choice(["bf16", "fp16", "fp32"]), widen=rng.random() < 0.5)
        if c["m"] * c["count"] * c["most"] <= 160000000:
            return c


# ----------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _sizes(c):
    """Elements per worker of each of the clip case's tensors: matrices and short vectors in turn."""
    return [c["most"] if j % 2 == 0 else max(1, c["most"] // 1000 + 7 * j) for j in range(c["count"])]


def prepare(case, seed):
    c, g = case, _generator(seed)
    dtype = _TYPES[c["dtype"]]
    s = dict(case)
    if c["op"] == "gated":
        m, T, D, F = c["m"], c["T"], c["D"], c["F"]
        s["x"] = _normal(g, (m, T, D), dtype)
        s["wg"] = _normal(g, (m, F, D), dtype, D ** -0.5)
        s["wu"] = _normal(g, (m, F, D), dtype, D ** -0.5)
        if c["train"]:
            s["dh"] = _normal(g, (m, T, F), dtype)
    elif c["op"] == "logprobs":
        N, V = c["N"], c["V"]
        s["logits"] = _normal(g, (N, V), dtype, 3.0)
        if c["masked"]:
            s["logits"].masked_fill_(torch.rand((N, V), generator=g, device="cuda") < 0.25, -math.inf)
        t = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        # the given token itself is never masked
        s["logits"].scatter_(1, t.long()[:, None], _normal(g, (N, 1), dtype, 3.0))
        # rows of padding at the end of sequences carry no token
        s["targets"] = torch.where(torch.rand((N,), generator=g, device="cuda") < 0.03, torch.full_like(t, -1), t)
        if c["train"]:
            s["dlogp"] = -torch.rand((N,), generator=g, device="cuda") / N
            s["dentropy"] = _normal(g, (N,), torch.float32, 0.01 / N)
    elif c["op"] == "embedding":
        m, T, V, D = c["m"], c["T"], c["V"], c["D"]
        s["table"] = _normal(g, (m, V, D), dtype)
        # few frequent tokens and many rare ones, and some padding
        u = torch.rand((m, T), generator=g, device="cuda")
        ids = ((V + 1.0) ** u - 1.0).to(torch.int32).clamp_(0, V - 1)
        s["ids"] = torch.where(torch.rand((m, T), generator=g, device="cuda") < 0.02, torch.full_like(ids, -1), ids)
        s["scale"] = float(D) ** 0.5
        if c["train"]:
            s["dout"] = _normal(g, (m, T, D), dtype)
    else:
        # every other worker's gradient is small enough to pass unclipped
        std = torch.where(torch.arange(c["m"], device="cuda") % 2 == 0, 1.0, 1e-4)[:, None]
        s["grads"] = [(torch.randn((c["m"], n), generator=g, device="cuda") * std).to(dtype) for n in _sizes(c)]
        s["out"] = [torch.empty_like(t, dtype=torch.float32 if c["widen"] else dtype) for t in s["grads"]]
        s["max_norm"] = 1.0
    return s


# -------------------------------------------------------------------------- one pass

def run(state):
    s = state
    if own:
        import paper_2002_09539_b200 as lib
        if s["op"] == "gated":
            if not s["train"]:
                return {"h": lib.gated_forward(s["x"], s["wg"], s["wu"], s["act"])}
            h, pre = lib.gated_forward(s["x"], s["wg"], s["wu"], s["act"], save=True)
            dx, dwg, dwu = lib.gated_backward(s["dh"], s["x"], s["wg"], s["wu"], pre, s["act"])
            return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}
        if s["op"] == "logprobs":
            r = lib.token_logprobs(s["logits"], s["targets"], s["top"])
            out = {"logp": r.logp, "entropy": r.entropy}
            if s["top"]:
                out["top_logp"], out["top_ids"] = r.top_logp, r.top_ids
            if s["train"]:
                out["dlogits"] = lib.token_logprobs_backward(s["dlogp"], s["dentropy"], s["logits"], s["targets"], r.stats, r.entropy)
            return out
        if s["op"] == "embedding":
            out = {"out": lib.embedding_forward(s["table"], s["ids"], s["scale"])}
            if s["train"]:
                out["dtable"] = lib.embedding_backward(s["dout"], s["ids"], s["V"], s["scale"])
            return out
        out, norms = lib.clip_grads(s["grads"], s["max_norm"], out=s["out"])
        return {"norms": norms, "out": out}
    return {"gated": _gated, "logprobs": _logprobs, "embedding": _embedding, "clip": _clip}[s["op"]](s)


def _activation(kind, a):
    """act(a) and its derivative."""
    if kind == "relu":
        return torch.clamp(a, min=0.0), (a > 0).to(a.dtype)
    if kind == "gelu":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (a + 0.044715 * a * a * a))
        return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)
    sig = 1.0 / (1.0 + torch.exp(-a))
    if kind == "sigmoid":
        return sig, sig * (1 - sig)
    return a * sig, sig * (1 + a * (1 - sig))


def _gated(s):
    dtype = s["x"].dtype
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    a, b = x @ wg.transpose(1, 2), x @ wu.transpose(1, 2)
    f, df = _activation(s["act"], a)
    out = {"h": (f * b).to(dtype)}
    if s["train"]:
        dh = s["dh"].float()
        da, db = dh * b * df, dh * f
        out["dx"] = (da @ wg + db @ wu).to(dtype)
        out["dwg"] = (da.transpose(1, 2) @ x).to(dtype)
        out["dwu"] = (db.transpose(1, 2) @ x).to(dtype)
    return out


def _logprobs(s):
    x, t = s["logits"].float(), s["targets"].long()
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    lp = x - lse
    p = e / total
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -plp.sum(dim=1)
    has = t >= 0
    at = torch.clamp(t, min=0)[:, None]
    out = {"logp": torch.where(has, lp.gather(1, at)[:, 0], torch.zeros_like(entropy)), "entropy": entropy}
    if s["top"]:
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_logp"] = v[:, : s["top"]] - lse
        out["top_ids"] = i[:, : s["top"]].to(torch.int32)
    if s["train"]:
        dlogp = torch.where(has, s["dlogp"], torch.zeros_like(s["dlogp"]))[:, None]
        d = -p * dlogp - s["dentropy"][:, None] * (plp + p * entropy[:, None])
        d.scatter_add_(1, at, dlogp)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _embedding(s):
    ids, V = s["ids"].long(), s["V"]
    m, T = ids.shape
    has = (ids >= 0)[..., None]
    flat = (torch.clamp(ids, min=0) + V * torch.arange(m, device=ids.device)[:, None]).reshape(-1)
    rows = s["table"].reshape(m * V, -1)[flat].reshape(m, T, -1).float() * s["scale"]
    out = {"out": torch.where(has, rows, torch.zeros_like(rows)).to(s["table"].dtype)}
    if s["train"]:
        d = s["dout"].float() * s["scale"]
        d = torch.where(has, d, torch.zeros_like(d))
        out["dtable"] = torch.zeros((m * V, d.shape[-1]), device=d.device).index_add_(0, flat, d.reshape(m * T, -1)).reshape(m, V, -1)
    return out


def _clip(s):
    sums = torch.stack([t.float().square().sum(dim=1) for t in s["grads"]]).sum(dim=0)
    norms = torch.sqrt(sums)
    c = torch.clamp(s["max_norm"] / (norms + 1e-6), max=1.0)[:, None]
    return {"norms": norms, "out": [(t.float() * c).to(o.dtype) for t, o in zip(s["grads"], s["out"])]}


# ------------------------------------------------------------------------------ work

def work(case):
    c = case
    e = 4 if c["dtype"] == "fp32" else 2
    if c["op"] == "gated":
        m, T, D, F = c["m"], c["T"], c["D"], c["F"]
        # forward: x, both weights in, h out; training adds dh in, dx and both weights' gradients out
        b = e * m * (T * D + 2 * F * D + T * F)
        f = 4 * m * T * D * F
        if c["train"]:
            b += e * m * (T * F + T * D + 2 * F * D)
            f += 8 * m * T * D * F
        return {"bytes": b, "flops": f}
    if c["op"] == "logprobs":
        n = c["N"] * c["V"]
        return {"bytes": n * e * (2 if c["train"] else 1) + c["N"] * (12 + 8 * c["top"] + (8 if c["train"] else 0)),
                "flops": n * (9 if c["train"] else 4)}
    if c["op"] == "embedding":
        m, T, V, D = c["m"], c["T"], c["V"], c["D"]
        # distinct rows of the table are read once: no more than V, no more than T
        b = m * (min(T, V) * D * e + T * D * e + 4 * T)
        if c["train"]:
            b += m * (T * D * e + V * D * 4)
        return {"bytes": b, "flops": m * T * D * (2 if c["train"] else 1)}
    n = c["m"] * sum(_sizes(c))
    return {"bytes": n * (e + (4 if c["widen"] else e)), "flops": 3 * n}


# ----------------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    if s["op"] == "gated":
        X, G, U = (s[k].double() for k in ("x", "wg", "wu"))
        a = torch.einsum("wtd,wfd->wtf", X, G)
        b = torch.einsum("wtd,wfd->wtf", X, U)
        k = s["act"]
        if k == "silu":
            y, dy = a * torch.sigmoid(a), torch.sigmoid(a) + a * torch.sigmoid(a) * torch.sigmoid(-a)
        elif k == "sigmoid":
            y, dy = torch.sigmoid(a), torch.sigmoid(a) * torch.sigmoid(-a)
        elif k == "relu":
            y, dy = torch.where(a > 0, a, 0.0), torch.where(a > 0, 1.0, 0.0)
        else:
            # 0.5 (1 + tanh z) = sigmoid(2 z)
            z2 = 2.0 * math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)
            y = a * torch.sigmoid(z2)
            dy = torch.sigmoid(z2) + a * torch.sigmoid(z2) * torch.sigmoid(-z2) * 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * a ** 2)
        out = {"h": y * b}
        if s["train"]:
            E = s["dh"].double()
            out["dx"] = torch.einsum("wtf,wfd->wtd", E * b * dy, G) + torch.einsum("wtf,wfd->wtd", E * y, U)
            out["dwg"] = torch.einsum("wtf,wtd->wfd", E * b * dy, X)
            out["dwu"] = torch.einsum("wtf,wtd->wfd", E * y, X)
        return out
    if s["op"] == "logprobs":
        x, t = s["logits"].double(), s["targets"].long()
        lse = torch.logsumexp(x, dim=1)
        p = torch.exp(x - lse[:, None])
        entropy = -torch.xlogy(p, p).sum(dim=1)
        rows = torch.arange(x.shape[0], device=x.device)
        picked = x[rows, t.clamp(min=0)] - lse
        out = {"logp": picked.masked_fill(t < 0, 0.0), "entropy": entropy}
        if s["top"]:
            v, i = torch.sort(x, dim=1, descending=True, stable=True)
            out["top_logp"] = v[:, : s["top"]] - lse[:, None]
            out["top_ids"] = i[:, : s["top"]].to(torch.int32)
        if s["train"]:
            dlp = s["dlogp"].double().masked_fill(t < 0, 0.0)
            onehot = torch.zeros_like(x)
            onehot[rows, t.clamp(min=0)] = 1.0
            d = dlp[:, None] * (onehot - p)
            d -= s["dentropy"].double()[:, None] * (torch.xlogy(p, p) + p * entropy[:, None])
            out["dlogits"] = d
        return out
    if s["op"] == "embedding":
        ids, W = s["ids"].long(), s["table"].double()
        has = (ids >= 0).double()[..., None]
        rows = torch.stack([W[i][ids[i].clamp(min=0)] for i in range(ids.shape[0])])
        out = {"out": rows * has * s["scale"]}
        if s["train"]:
            d = s["dout"].double() * has * s["scale"]
            out["dtable"] = torch.stack([torch.zeros_like(W[i]).index_add_(0, ids[i].clamp(min=0), d[i]) for i in range(ids.shape[0])])
        return out
    whole = torch.cat([t.double() for t in s["grads"]], dim=1)
    norms = torch.linalg.vector_norm(whole, dim=1)
    c = torch.minimum(torch.ones_like(norms), s["max_norm"] / (norms + 1e-6))[:, None]
    return {"norms": norms, "out": [t.double() * c for t in s["grads"]]}
