"""What is measured of the operators around a model's experts and its answers: the router with the
sort of its tokens by expert and its gradient, rows taken to the experts and back with their
gradients, the norm of all gradients and clipping by it, and drafted tokens verified against the
target's probabilities.

Each operator has a plain form here, of elementary torch operations in 32 bits (64 for long sums and
for values next to a border), rounded once at the end.  With ``own`` set, ``run`` makes the calls a
user makes of paper_1903_05133_gb300.operators.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
NONE = -1e30                    # logits at or below it are a mask's
ACCEPTED = 0.85                 # of the drafts, as prepare() makes them: about


# ---------------------------------------------------------------------- the cases
def listed():
    return [
        # Answering: a batch of 8 single tokens and the router of one layer.
        dict(name="route: single tokens", op="route", rows=8, experts=64, k=6, dtype="fp32", over="chosen", learners=0),
        # The router of a training batch with its sort, 32-bit logits.
        dict(name="route: training batch", op="route", rows=16384, experts=128, k=8, dtype="fp32", over="chosen",
             learners=0),
        # The gradient of a router whose weights are probabilities among all experts, 16 learners of 60
        # experts (an odd width for the warps), each on its own rows.
        dict(name="route: gradient", op="route_grad", rows=20000, experts=60, k=4, dtype="bf16", over="all", learners=16),
        # The rows of a training batch to their experts.
        dict(name="dispatch: training batch", op="dispatch", rows=8192, k=4, width=4096, experts=64, dtype="bf16",
             dropped=False),
        # Their gradient at an odd width, which suits no wide load, with tokens that found no expert.
        dict(name="dispatch: gradient, odd", op="dispatch_grad", rows=3001, k=3, width=1111, experts=33, dtype="fp16",
             dropped=True),
        # Answering: the experts' results of 8 single tokens.
        dict(name="combine: single tokens", op="combine", rows=8, k=6, width=4096, experts=64, dtype="bf16", out="bf16",
             dropped=False),
        # The experts' results of a training batch.
        dict(name="combine: training batch", op="combine", rows=8192, k=4, width=4096, experts=64, dtype="bf16",
             out="bf16", dropped=False),
        # Its gradient, the weights' among it.
        dict(name="combine: gradient", op="combine_grad", rows=8192, k=4, width=4096, experts=64, dtype="bf16",
             out="bf16", dropped=False),
        # The norms of four learners' gradients, one a learner, and the scales that clip them.
        dict(name="norm: four learners", op="norm", grad="bf16", dims="12288-4096-4096-1000", learners=4),
        # One norm over 300 small tensors of odd sizes, clipped in place.
        dict(name="clip: many small tensors", op="clip", grad="fp32", tensors=300, most=30000, learners=0),
        # One sequence's four drafts: answering.
        dict(name="verify: one sequence", op="verify", sequences=1, drafts=4, classes=128001, dtype="bf16", probs="fp32",
             mask=False, temperature=1.0),
        # A batch under a mask, 32-bit logits, odd length, some sequences with fewer drafts.
        dict(name="verify: batch", op="verify", sequences=128, drafts=5, classes=50021, dtype="fp32", probs="fp32",
             mask=True, temperature=0.8),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "dispatch", "dispatch_grad", "combine", "combine", "combine_grad",
                     "norm", "clip", "verify", "verify"])
    if op.startswith("route"):
        learners = rng.choice([0, 0, _log(rng, 2, 16)])
        experts = _log(rng, 4, 1024 // max(learners, 1))
        return dict(op=op, rows=_log(rng, 1, 32768), experts=experts, k=rng.randint(1, min(experts, 16)),
                    dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]), over=rng.choice(["chosen", "all"]),
                    learners=learners)
    if op.split("_")[0] in ("dispatch", "combine"):
        while True:
            c = dict(op=op, rows=_log(rng, 1, 16384), k=rng.randint(1, 8), width=_log(rng, 8, 8192),
                     experts=_log(rng, 8, 256), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                     dropped=rng.random() < 0.3)
            if rng.random() < 0.7:      # most widths are multiples of 8
                c["width"] = -(-c["width"] // 8) * 8
            if op.startswith("combine"):
                c["out"] = rng.choice([c["dtype"], c["dtype"], "fp32"])
            if work(c)["bytes"] < 6e8:
                return c
    if op in ("norm", "clip"):
        return dict(op=op, grad=rng.choice(["bf16", "fp16", "fp32"]), tensors=_log(rng, 1, 400),
                    most=_log(rng, 100, 200000), learners=rng.choice([0, 0, _log(rng, 1, 16)]))
    while True:
        c = dict(op=op, sequences=_log(rng, 1, 256), drafts=rng.randint(1, 8), classes=_log(rng, 100, 150000),
                 dtype=rng.choice(["bf16", "fp16", "fp32"]), probs=rng.choice(["fp32", "fp32", "bf16", "none"]),
                 mask=rng.random() < 0.3, temperature=rng.choice([1.0, round(rng.uniform(0.5, 1.5), 2)]))
        if c["sequences"] * (c["drafts"] + 1) * c["classes"] < 3.8e7:
            return c


# ---------------------------------------------------------------------- sizes
def _shapes(case):
    """The shapes of the gradients; with learners their first dimension is the learner."""
    P = case["learners"]
    if "dims" in case:
        dims = [int(d) for d in case["dims"].split("-")]
        return [s for i, o in zip(dims[:-1], dims[1:]) for s in ((P, o, i), (P, o))]
    r = random.Random(case["tensors"] * 1000003 + case["most"])
    sizes = [r.randint(1, case["most"]) for _ in range(case["tensors"])]
    return [(P, -(-n // P)) if P else (n,) for n in sizes]


def work(case):
    op = case["op"]
    if op == "route":
        T, E, k = case["rows"], case["experts"], case["k"]
        return {"bytes": T * E * SIZE[case["dtype"]] + T * (16 * k + 4) + 4 * E * max(case["learners"], 1),
                "flops": 4 * T * E}
    if op == "route_grad":
        T, E, k = case["rows"], case["experts"], case["k"]
        b = T * E * SIZE[case["dtype"]] + 12 * T * k
        if case["over"] == "all":
            b += T * E * SIZE[case["dtype"]] + 4 * T
        return {"bytes": b, "flops": 4 * T * (E if case["over"] == "all" else k)}
    if op.split("_")[0] in ("dispatch", "combine"):
        T, R, D, e = case["rows"], case["rows"] * case["k"], case["width"], SIZE[case["dtype"]]
        if op in ("dispatch", "dispatch_grad"):
            return {"bytes": (T + R) * D * e + 4 * R, "flops": 0 if op == "dispatch" else R * D}
        o = SIZE[case["out"]]
        if op == "combine":
            return {"bytes": T * D * o + R * D * e + 8 * R, "flops": 2 * R * D}
        return {"bytes": T * D * o + 2 * R * D * e + 12 * R, "flops": 3 * R * D}
    if op in ("norm", "clip"):
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": n * SIZE[case["grad"]] * (1 if op == "norm" else 2), "flops": (2 if op == "norm" else 3) * n}
    B, K, V = case["sequences"], case["drafts"], case["classes"]
    rows = sum(ACCEPTED ** i for i in range(K + 1))          # those behind a rejected draft are not needed
    one = SIZE[case["dtype"]] + (1 if case["mask"] else 0)
    last = 4 + (0 if case["probs"] == "none" else SIZE[case["probs"]])
    return {"bytes": int(B * V * (rows * one + last)), "flops": int(B * V * (3 * rows + 5))}


# ---------------------------------------------------------------------- inputs
def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype).mul_(std)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _router(gen, rows, experts, dtype):
    """Logits of experts that are not equally liked."""
    return (_normal(gen, rows, experts) + _normal(gen, experts, std=0.5)).to(dtype)


def _learners(case, seed):
    """Where each learner's rows begin: batches of different sizes, one after the other."""
    P, T = case["learners"], case["rows"]
    if not P:
        return None
    r = np.random.default_rng(seed)
    p = np.exp(0.4 * r.standard_normal(P))
    return torch.tensor(np.concatenate([[0], np.cumsum(r.multinomial(T, p / p.sum()))]), dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    op = case["op"]
    s = {"op": op, "case": case}
    if op.startswith("route"):
        s["logits"] = _router(gen, case["rows"], case["experts"], DTYPES[case["dtype"]])
        s["learners"] = _learners(case, seed)
        if op == "route_grad":
            f = _plain_route(s)
            s |= {n: f[n] for n in ("experts", "weights", "lse")}
            s["dweights"] = _normal(gen, case["rows"], case["k"])
        return s
    if op.split("_")[0] in ("dispatch", "combine"):
        T, k, D, E = case["rows"], case["k"], case["width"], case["experts"]
        z = _router(gen, T, E, torch.float32)
        best, experts = torch.sort(z, dim=1, descending=True, stable=True)
        experts = experts[:, :k].to(torch.int32)
        if case["dropped"]:
            experts = torch.where(_uniform(gen, T, k) < 0.1, -1, experts)
        s["weights"] = torch.softmax(best[:, :k], dim=1)
        s["offsets"], s["place"], _ = _plain_sort(experts, E)
        dt = DTYPES[case["dtype"]]
        if op == "dispatch":
            s["x"] = _normal(gen, T, D, dtype=dt)
        elif op == "dispatch_grad":
            s["dxs"] = _normal(gen, T * k, D, dtype=dt)
        else:
            s["y"] = _normal(gen, T * k, D, dtype=dt)
            if op == "combine_grad":
                s["dout"] = _normal(gen, T, D, dtype=DTYPES[case["out"]])
        return s
    if op in ("norm", "clip"):
        P, shapes = case["learners"], _shapes(case)
        size = 1e-3 * torch.exp(_normal(gen, max(P, 1), std=0.5))
        ends = np.cumsum([math.prod(shape) for shape in shapes]).tolist()
        n = ends[-1]
        # all gradients in one buffer, one directly after the other
        s["flat"] = _normal(gen, n, dtype=DTYPES[case["grad"]])
        s["grads"] = [s["flat"][e - math.prod(shape):e].view(shape) for shape, e in zip(shapes, ends)]
        for g in s["grads"]:
            g.mul_(size.view(-1, *[1] * (g.dim() - 1)) if P else size[0])
        # about half of the learners are over the largest norm; one norm for all always is
        s["max_norm"] = 1e-3 * math.sqrt(n / P) if P else 0.5 * size[0].item() * math.sqrt(n)
        return s
    B, K, V = case["sequences"], case["drafts"], case["classes"]
    z = _normal(gen, B, K + 1, V, std=2.0)
    sure = torch.randint(0, V, (B, K + 1, 1), generator=gen, device="cuda")
    # a model that is sure of two positions in three
    z.scatter_(2, sure, math.log(V) + 4.0 - 4.0 * (_uniform(gen, B, K + 1, 1) < 0.35))
    s["allowed"] = None
    if case["mask"]:
        s["allowed"] = _uniform(gen, B, K + 1, V) < 0.5
        s["allowed"].scatter_(2, sure, True)
    # the draft's own model is off by a little
    d = (z[:, :K] + _normal(gen, B, K, V, std=0.8)) / case["temperature"]
    if s["allowed"] is not None:
        d = torch.where(s["allowed"][:, :K], d, -math.inf)
    q = torch.exp(d - d.amax(2, keepdim=True))
    q = q / q.sum(2, keepdim=True)
    if case["probs"] == "none":
        x = q.argmax(2)                             # a draft model that takes its likeliest token
        s["probs"] = None
    else:
        x = (q / torch.empty_like(q).exponential_(generator=gen)).argmax(2)
        s["probs"] = q.to(DTYPES[case["probs"]])
    # a sequence in eight has fewer drafts
    fewer = torch.where(_uniform(gen, B, 1) < 0.125, (_uniform(gen, B, 1) * K).long(), K)
    s["drafts"] = torch.where(torch.arange(K, device="cuda") < fewer, x, -1).to(torch.int32)
    s["logits"] = z.to(DTYPES[case["dtype"]])
    s["uniform"] = _uniform(gen, B, K)
    s["noise"] = torch.empty(B, V, device="cuda").exponential_(generator=gen)
    return s


# ---------------------------------------------------------------------- plain forms
def _plain_sort(groups, G):
    """Entries [rows, k] by group, stable; what has no group in [0, G) has no place."""
    g = groups.reshape(-1).long()
    inside = (g >= 0) & (g < G)
    key = torch.where(inside, g, G)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(len(order), device=g.device)
    offsets = torch.searchsorted(key[order], torch.arange(G + 1, device=g.device))
    count = inside.sum()
    source = torch.where(torch.arange(len(order), device=g.device) < count, order, -1)
    place = torch.where(inside, place, -1)
    return offsets.int(), place.view(groups.shape).int(), source.int()


def _plain_route(s):
    c = s["case"]
    z = s["logits"].float()
    z = torch.where(z <= NONE, -math.inf, z)
    best, experts = torch.sort(z, dim=1, descending=True, stable=True)
    best, experts = best[:, :c["k"]], experts[:, :c["k"]]
    m = best[:, :1]
    m = torch.where(m == -math.inf, 0.0, m)
    total = torch.exp(z - m).sum(1, keepdim=True)
    e = torch.exp(best - m)
    weights = e / (e.sum(1, keepdim=True) if c["over"] == "chosen" else total)
    none = best == -math.inf
    experts = torch.where(none, -1, experts).int()
    group, G = experts, c["experts"]
    if s["learners"] is not None:
        t = torch.arange(z.shape[0], device=z.device, dtype=torch.int32)
        learner = torch.searchsorted(s["learners"][1:].contiguous(), t, right=True).int()
        group = torch.where(experts < 0, -1, experts + learner[:, None] * G)
        G = G * c["learners"]
    offsets, place, source = _plain_sort(group, G)
    return {"experts": experts, "weights": torch.where(none, 0.0, weights), "lse": (m + torch.log(total))[:, 0],
            "offsets": offsets, "place": place, "source": source}


def _plain_route_grad(s):
    c = s["case"]
    w, dw = s["weights"], s["dweights"]
    mean = (w * dw).sum(1, keepdim=True)
    one = s["experts"].clamp(min=0).long()
    if c["over"] == "chosen":
        dz = torch.zeros(s["logits"].shape, device=w.device)
        dz.scatter_add_(1, one, torch.where(s["experts"] < 0, 0.0, w * (dw - mean)))
    else:
        dz = -mean * torch.exp(s["logits"].float() - s["lse"][:, None])
        dz.scatter_add_(1, one, torch.where(s["experts"] < 0, 0.0, w * dw))
    return dz.to(s["logits"].dtype)


def _plain_dispatch(s):
    place = s["place"].reshape(-1).long()
    T, k = s["place"].shape
    inside = place >= 0
    xs = torch.zeros(T * k, s["x"].shape[1], dtype=s["x"].dtype, device=place.device)
    xs[place[inside]] = s["x"][torch.arange(T * k, device=place.device)[inside] // k]
    return xs


def _taken(rows, place):
    """[T, k, D] in 32 bits: the rows at their tokens' places, zeros where there is none."""
    at = rows.float()[place.clamp(min=0).long()]
    return torch.where(place[..., None] < 0, 0.0, at)


def _plain_dispatch_grad(s):
    return _taken(s["dxs"], s["place"]).sum(1).to(s["dxs"].dtype)


def _plain_combine(s):
    w = s["weights"][..., None]
    return (_taken(s["y"], s["place"]) * w).sum(1).to(DTYPES[s["case"]["out"]])


def _plain_combine_grad(s):
    place = s["place"].reshape(-1).long()
    inside = place >= 0
    d = s["dout"].float()[:, None]
    dy = torch.zeros_like(s["y"])
    dy[place[inside]] = (d * s["weights"][..., None]).flatten(0, 1)[inside].to(dy.dtype)
    return {"dy": dy, "dweights": (_taken(s["y"], s["place"]) * d).sum(2)}


def _plain_norm(s):
    P = s["case"]["learners"]
    total = 0
    for g in s["grads"]:
        total = total + g.float().view(max(P, 1), -1).square().sum(1).double()
    norm = torch.sqrt(total)
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
    if s["op"] == "norm":
        return {"norm": norm.float(), "scale": scale}
    for g in s["grads"]:
        g.copy_(g.float() * (scale.view(-1, *[1] * (g.dim() - 1)) if P else scale))
    return {"norm": norm.float(), "scale": scale, "grads": s["flat"]}


def _plain_verify(s):
    c = s["case"]
    z = s["logits"].double() / c["temperature"]
    out = s["logits"] <= NONE
    if s["allowed"] is not None:
        out = out | ~s["allowed"]
    z = torch.where(out, -math.inf, z)
    m = z.amax(2, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(2, keepdim=True))
    B, K = s["drafts"].shape
    x = s["drafts"].long()
    given = x.clamp(min=0)[..., None]
    p = torch.exp(z[:, :K].gather(2, given) - lse[:, :K])[..., 0]
    q = torch.ones_like(p) if s["probs"] is None else s["probs"].gather(2, given)[..., 0].double()
    ok = (x >= 0) & (s["uniform"].double() * q < p)
    n = ok.long().cumprod(1).sum(1)                          # drafts before the first that fails
    b = torch.arange(B, device=n.device)
    rejected = (n < K) & (x[b, n.clamp(max=K - 1)] >= 0)
    last = torch.exp(z[b, n] - lse[b, n])
    at = n.clamp(max=K - 1)
    if s["probs"] is None:
        r = last.clone()
        r[b, x[b, at].clamp(min=0)] = 0.0
    else:
        r = (last - s["probs"][b, at].double()).clamp(min=0)
    r = torch.where((rejected & (r > 0).any(1))[:, None], r, last)
    token = (r / s["noise"].double()).argmax(1)
    i = torch.arange(K + 1, device=n.device)
    tokens = torch.where(i < n[:, None], torch.nn.functional.pad(x, (0, 1)), -1)
    tokens[b, n] = token
    logp = torch.where(tokens < 0, 0.0, (z - lse).gather(2, tokens.clamp(min=0)[..., None])[..., 0])
    return {"tokens": tokens.int(), "accepted": n.int(), "logp": logp.float()}


# ---------------------------------------------------------------------- one pass
PLAIN = {"route": _plain_route, "route_grad": _plain_route_grad, "dispatch": _plain_dispatch,
         "dispatch_grad": _plain_dispatch_grad, "combine": _plain_combine, "combine_grad": _plain_combine_grad,
         "norm": _plain_norm, "clip": _plain_norm, "verify": _plain_verify}


def run(s):
    op, c = s["op"], s["case"]
    if not own:
        return PLAIN[op](s)
    from paper_1903_05133_gb300 import operators as ops
    if op == "route":
        return ops.route(s["logits"], c["k"], over=c["over"], learners=s["learners"])._asdict()
    if op == "route_grad":
        return ops.route_backward(s["dweights"], s["logits"], s["experts"], s["weights"], lse=s["lse"], over=c["over"])
    if op == "dispatch":
        return ops.dispatch(s["x"], s["place"], s["offsets"])
    if op == "dispatch_grad":
        return ops.dispatch_backward(s["dxs"], s["place"])
    if op == "combine":
        return ops.combine(s["y"], s["place"], s["weights"], out_dtype=DTYPES[c["out"]])
    if op == "combine_grad":
        dy, dweights = ops.combine_backward(s["dout"], s["y"], s["place"], s["weights"], s["offsets"])
        return {"dy": dy, "dweights": dweights}
    learners = c.get("learners") or None
    if op == "norm":
        return ops.grad_norm(s["grads"], max_norm=s["max_norm"], learners=learners)._asdict()
    if op == "clip":
        r = ops.clip_gradients(s["grads"], s["max_norm"], learners=learners)
        return {"norm": r.norm, "scale": r.scale, "grads": s["flat"]}
    r = ops.verify_drafts(s["logits"], s["drafts"], s["uniform"], s["noise"], draft_probs=s["probs"],
                          temperature=c["temperature"], allowed=s["allowed"])
    return {"tokens": r.tokens, "accepted": r.accepted, "logp": r.logp}


# ---------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    h = lambda a: a.double().cpu().numpy()  # noqa: E731
    if op == "route":
        z = h(s["logits"])
        best = -np.sort(-z, axis=1)[:, :case["k"]]
        m = best[:, :1]
        total = np.exp(z - m).sum(1, keepdims=True)
        e = np.exp(best - m)
        return {"experts": None, "weights": e / (e.sum(1, keepdims=True) if case["over"] == "chosen" else total),
                "lse": (m + np.log(total))[:, 0], "offsets": None, "place": None, "source": None}
    if op == "route_grad":
        # the logits' gradient of sum(dw w): w = e^z over the sum of the chosen, or of all
        z, dw, at = h(s["logits"]), h(s["dweights"]), s["experts"].cpu().numpy().astype(np.int64)
        e = np.exp(z - z.max(1, keepdims=True))
        chosen = np.zeros(z.shape, bool)
        np.put_along_axis(chosen, at, True, 1)
        p = np.where(chosen | (case["over"] == "all"), e, 0.0)
        p /= p.sum(1, keepdims=True)
        up = np.zeros(z.shape)
        np.put_along_axis(up, at, dw, 1)
        return p * (up - (p * up).sum(1, keepdims=True))
    if op in ("dispatch", "dispatch_grad", "combine", "combine_grad"):
        return _exact_rows(s, case)
    if op in ("norm", "clip"):
        P = case["learners"]
        total = np.zeros(max(P, 1))
        for g in s["grads"]:
            for i in range(max(P, 1)):
                a = (g[i] if P else g).double()
                total[i] += float((a * a).sum())
        norm = np.sqrt(total)
        scale = np.minimum(1.0, s["max_norm"] / norm)
        out = {"norm": norm, "scale": scale}
        if op == "clip":
            out["grads"] = np.concatenate([(h(g) * scale.reshape(-1, *[1] * (g.dim() - 1)) if P else h(g) * scale[0]).reshape(-1)
                                           for g in s["grads"]])
        return out
    return _exact_verify(s, case)


def _exact_rows(s, case):
    op, T, k, D = case["op"], case["rows"], case["k"], case["width"]
    place = s["place"].cpu().numpy()
    if op == "dispatch":
        xs = np.zeros((T * k, D))
        x = s["x"].double().cpu().numpy()
        for j in range(k):
            has = place[:, j] >= 0
            xs[place[has, j]] = x[has]
        return xs
    rows = s["dxs"] if op == "dispatch_grad" else s["y"]
    out = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    dy, dw = (torch.zeros(T * k, D, dtype=torch.float64, device="cuda"), np.zeros((T, k))) if op == "combine_grad" else (None, None)
    for j in range(k):
        t = torch.nonzero(s["place"][:, j] >= 0)[:, 0]
        at = s["place"][t, j].long()
        r = rows[at].double()
        w = s["weights"][t, j].double()[:, None]
        if op == "combine_grad":
            d = s["dout"][t].double()
            dy[at] = w * d
            dw[t.cpu().numpy(), j] = (r * d).sum(1).cpu().numpy()
        else:
            out[t] += r if op == "dispatch_grad" else w * r
    return {"dy": dy.cpu().numpy(), "dweights": dw} if op == "combine_grad" else out.cpu().numpy()


def _exact_verify(s, case):
    """Sequence by sequence, as the rule says it."""
    B, K = s["drafts"].shape
    drafts, u = s["drafts"].tolist(), s["uniform"].tolist()
    logp = np.zeros((B, K + 1))
    for b in range(B):
        n, rejected = 0, False
        while True:
            z = s["logits"][b, n].double() / case["temperature"]
            if s["allowed"] is not None:
                z = z.masked_fill(~s["allowed"][b, n], -math.inf)
            lp = torch.log_softmax(z, 0)
            if n == K or drafts[b][n] < 0:
                break
            x = drafts[b][n]
            q = 1.0 if s["probs"] is None else s["probs"][b, n, x].item()
            if not u[b][n] * q < math.exp(lp[x].item()):
                rejected = True
                break
            logp[b, n] = lp[x].item()
            n += 1
        p = torch.exp(lp)
        if rejected:
            r = p.clone()
            if s["probs"] is None:
                r[drafts[b][n]] = 0
            else:
                r = torch.clamp(p - s["probs"][b, n].double(), min=0)
            p = r if bool((r > 0).any()) else p
        logp[b, n] = lp[torch.argmax(p / s["noise"][b].double())].item()
    return {"tokens": None, "accepted": None, "logp": logp}
