"""What is measured of the operators for models with grouped weights: products grouped by expert
or learner (forward and both gradients), log probabilities of given tokens (forward and gradient),
and the AdamW step over many tensors.

Each operator has a plain form here, of elementary torch operations in 32 bits, rounded once at the
end.  With ``own`` set, ``run`` makes the calls a user makes of paper_1903_05133_gb300.operators.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BLOCK = 256                     # elements that share one scale of the 8-bit AdamW states
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8


# ---------------------------------------------------------------------- the cases
def listed():
    return [
        # One token for each of 32 experts (or learners) of 4096 -> 4096: answering, where the
        # weights' bytes are all that counts.
        dict(name="product: one row each", op="product", groups=32, rows=32, inner=4096, outer=4096,
             dtype="bf16", out="bf16", relu=False, bias=False),
        # The hidden layer of 32 learners on ragged batches, with its bias and ReLU.
        dict(name="product: ragged batches", op="product", groups=32, rows=16384, inner=4096,
             outer=4096, dtype="bf16", out="bf16", relu=True, bias=True),
        # The gradient of the rows of 64 learners' 2048 -> 2048 layer, through the ReLU below it.
        dict(name="product: gradient of rows", op="product_dx", groups=64, rows=8192, inner=2048,
             outer=2048, dtype="fp16", out="fp16", relu=True),
        # The weights' gradient of the 4096 -> 4096 layer on ragged batches, with the bias's.
        dict(name="product: gradient of weights", op="product_dw", groups=32, rows=16384, inner=4096,
             outer=4096, dtype="bf16", out="bf16", bias=True),
        # A small layer onto 10 classes, whose rows of 20 bytes suit no wide load, in 32 bits.
        dict(name="product: small, odd, 32 bits", op="product_dw", groups=16, rows=500, inner=512,
             outer=10, dtype="bf16", out="fp32", bias=True),
        # One row of a large vocabulary, with its 20 likeliest tokens: answering.
        dict(name="logprobs: one row", op="logprobs", rows=1, classes=128001, dtype="bf16", top=20,
             mask=False, temperature=1.0),
        # Scoring a batch under a mask that leaves some rows empty, 32-bit logits, odd length.
        dict(name="logprobs: masked rows", op="logprobs", rows=96, classes=50021, dtype="fp32", top=8,
             mask=True, temperature=0.7),
        # The loss of a training batch.
        dict(name="logprobs: training batch", op="logprobs", rows=8192, classes=32768, dtype="bf16",
             top=0, mask=False, temperature=1.0),
        # Its gradient, with the entropy's.
        dict(name="logprobs: gradient", op="logprobs_grad", rows=8192, classes=32768, dtype="bf16",
             mask=False, temperature=1.0, entropy=True),
        # One learner of 12288-4096-4096-1000 with 32-bit states and a bf16 copy of its weights.
        dict(name="adamw: 32-bit states", op="adamw", bits=32, grad="fp32", copy="bf16",
             dims="12288-4096-4096-1000", learners=1, scale=False),
        # Four of them with 8-bit states and bf16 gradients under a clipping scale.
        dict(name="adamw: 8-bit states", op="adamw", bits=8, grad="bf16", copy="bf16",
             dims="12288-4096-4096-1000", learners=4, scale=True),
        # 300 small tensors of odd sizes: biases, norms, small projections.
        dict(name="adamw: many small tensors", op="adamw", bits=8, grad="fp32", copy="none", tensors=300,
             most=30000, scale=False),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["product", "product", "product_dx", "product_dw", "product_dw", "logprobs", "logprobs",
                     "logprobs_grad", "adamw", "adamw"])
    if op.startswith("product"):
        while True:
            c = dict(op=op, groups=_log(rng, 1, 64), rows=_log(rng, 1, 16384), inner=_log(rng, 64, 4500),
                     outer=_log(rng, 8, 4500), dtype=rng.choice(["bf16", "fp16"]))
            if rng.random() < 0.7:      # most layers' widths are multiples of 8
                c["inner"], c["outer"] = -(-c["inner"] // 8) * 8, -(-c["outer"] // 8) * 8
            c["out"] = rng.choice([c["dtype"], "fp32"])
            if op == "product":
                c["relu"], c["bias"] = rng.random() < 0.5, rng.random() < 0.5
            elif op == "product_dx":
                c["relu"] = rng.random() < 0.5
            else:
                c["bias"] = rng.random() < 0.5
            w = work(c)
            if w["flops"] < 2.5e11 and w["bytes"] < 1.5e9:
                return c
    if op.startswith("logprobs"):
        while True:
            c = dict(op=op, rows=_log(rng, 1, 8192), classes=_log(rng, 10, 150000),
                     dtype=rng.choice(["bf16", "fp16", "fp32"]), mask=rng.random() < 0.3,
                     temperature=rng.choice([1.0, round(rng.uniform(0.3, 2.0), 2)]))
            if op == "logprobs":
                c["top"] = rng.choice([0, rng.randint(1, 32)])
            else:
                c["entropy"] = rng.random() < 0.5
            if work(c)["bytes"] < 8e8:
                return c
    c = dict(op=op, bits=rng.choice([8, 32]), grad=rng.choice(["bf16", "fp16", "fp32"]),
             copy=rng.choice(["bf16", "fp16", "none"]), scale=rng.random() < 0.5)
    c["tensors"], c["most"] = _log(rng, 1, 400), _log(rng, 100, 200000)
    return c


# ---------------------------------------------------------------------- sizes
def _shapes(case):
    """The sizes of an AdamW case's tensors and whether each is decayed."""
    if "dims" in case:
        dims = [int(d) for d in case["dims"].split("-")]
        one = [(n, d) for i, o in zip(dims[:-1], dims[1:]) for n, d in ((i * o, True), (o, False))]
        return one * case["learners"]
    r = random.Random(case["tensors"] * 1000003 + case["most"])
    return [(r.randint(1, case["most"]), r.random() < 0.7) for _ in range(case["tensors"])]


def _nonempty(case):
    return min(case["rows"], case["groups"] - case["groups"] // 16)


def work(case):
    op = case["op"]
    if op.startswith("product"):
        G, T, K, N = (case[k] for k in ("groups", "rows", "inner", "outer"))
        e, o = SIZE[case["dtype"]], SIZE[case["out"]]
        if op == "product":
            b = T * K * e + _nonempty(case) * N * (K * e + (4 if case["bias"] else 0)) + T * N * o
        elif op == "product_dx":
            b = T * N * e + _nonempty(case) * N * K * e + T * K * (o + (e if case["relu"] else 0))
        else:
            b = T * (K + N) * e + G * N * (K * o + (4 if case["bias"] else 0))
        return {"bytes": b, "flops": 2 * T * K * N}
    if op.startswith("logprobs"):
        T, V, e = case["rows"], case["classes"], SIZE[case["dtype"]]
        b = T * V * (e + (1 if case["mask"] else 0))
        if op == "logprobs":
            return {"bytes": b + T * (16 + 8 * case["top"]), "flops": 6 * T * V}
        return {"bytes": b + T * V * e + T * 20, "flops": 6 * T * V}
    n = sum(s for s, _ in _shapes(case))
    c = 0 if case["copy"] == "none" else SIZE[case["copy"]]
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + SIZE[case["grad"]] + c + state), "flops": 14 * n}


# ---------------------------------------------------------------------- inputs
def _group_sizes(case, seed):
    """Rows of each group: a sixteenth of the groups empty, the others uneven."""
    r = np.random.default_rng(seed)
    G, T, full = case["groups"], case["rows"], _nonempty(case)
    sizes = np.zeros(G, np.int64)
    if full:
        at = r.permutation(G)[:full]
        p = np.exp(0.4 * r.standard_normal(full))
        sizes[at] = 1 + r.multinomial(T - full, p / p.sum())
    return sizes


def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    # in 16 bits directly where the result is: the inputs of the large cases fill gigabytes
    return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype).mul_(std)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    op = case["op"]
    s = {"op": op, "case": case}
    if op.startswith("product"):
        G, T, K, N = (case[k] for k in ("groups", "rows", "inner", "outer"))
        dt = DTYPES[case["dtype"]]
        sizes = _group_sizes(case, seed)
        s["rows_max"] = int(sizes.max())
        s["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
        if op != "product_dw":
            s["w"] = _normal(gen, G, N, K, std=math.sqrt(2 / K), dtype=dt)
        if op != "product_dx":
            s["x"] = _normal(gen, T, K, dtype=dt)
        if op != "product":
            s["dy"] = _normal(gen, T, N, std=0.05, dtype=dt)
        if op == "product":
            s["bias"] = _normal(gen, G, N, std=0.1) if case["bias"] else None
        if op == "product_dx":
            s["h"] = _normal(gen, T, K, dtype=dt).relu_() if case["relu"] else None
        return s
    if op.startswith("logprobs"):
        T, V, dt = case["rows"], case["classes"], DTYPES[case["dtype"]]
        z = _normal(gen, T, V, std=2.0, dtype=dt)
        t = torch.randint(0, V, (T,), generator=gen, device="cuda")
        z[torch.arange(T, device="cuda"), t] += 6.0        # a model that has learnt something
        s["logits"] = z
        s["targets"] = torch.where(torch.rand(T, generator=gen, device="cuda") < 0.05, -1, t).to(torch.int32)
        s["allowed"] = None
        if case["mask"]:
            s["allowed"] = torch.rand(T, V, generator=gen, device="cuda") < 0.3
            s["allowed"][torch.arange(T, device="cuda") % 32 == 5] = False
        if op == "logprobs_grad":
            f = _plain_logprobs(z, s["targets"], s["allowed"], case["temperature"], 0)
            s["lse"], s["entropy"] = f["lse"], f["entropy"]
            s["dlogp"] = _normal(gen, T, std=1.0) / T - 1.0 / T
            s["dentropy"] = _normal(gen, T, std=0.01) / T if case["entropy"] else None
        return s
    shapes = _shapes(case)
    ends = np.cumsum([-(-n // BLOCK) * BLOCK for n, _ in shapes])
    starts = np.concatenate([[0], ends[:-1]])
    total = int(ends[-1])
    real = torch.zeros(total, dtype=torch.bool, device="cuda")
    s["decay"] = torch.zeros(total // BLOCK, 1, device="cuda")
    for (n, d), at, end in zip(shapes, starts.tolist(), ends.tolist()):
        real[at:at + n] = True
        if d:
            s["decay"][at // BLOCK:end // BLOCK] = 0.1
    s["p"] = _normal(gen, total, std=0.02).mul_(real)
    s["g"] = _normal(gen, total, std=1e-3, dtype=DTYPES[case["grad"]]).mul_(real)
    s["copy"] = None if case["copy"] == "none" else s["p"].to(DTYPES[case["copy"]])
    s["t"], s["lr"], s["seed"] = 100, 1e-3, seed
    s["scale"] = torch.rand(1, generator=gen, device="cuda") + 0.5 if case["scale"] else None
    m = _normal(gen, total, std=3e-4).mul_(real)
    v = (_normal(gen, total, std=1e-3).square_() + 1e-7).mul_(real)
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _to_8(m)
        s["root"], s["root_scale"] = _to_8(v.sqrt_())
    del m, v, real
    cut = lambda a: [a[at:at + n] for (n, _), at in zip(shapes, starts.tolist())]  # noqa: E731
    s["grads"] = cut(s["g"])
    if own:
        from paper_1903_05133_gb300.operators import AdamW
        o = AdamW(cut(s["p"]), bits=case["bits"], beta1=BETA1, beta2=BETA2, eps=EPS,
                  decay=[0.1 if d else 0.0 for _, d in shapes],
                  copies=None if s["copy"] is None else cut(s["copy"]))
        o.load_state_dict({"t": s["t"], **{k: s[k] for k in ("m", "v", "m_scale", "root", "root_scale") if k in s}})
        s["opt"] = o
    return s


# ---------------------------------------------------------------------- plain forms
def _padded(a, offsets, rows_max):
    """[G, rows_max, ...] in 32 bits with zeros after each group's rows."""
    at = offsets[:-1, None].long() + torch.arange(rows_max, device=a.device)
    inside = at < offsets[1:, None]
    return a.float()[at.clamp(max=max(a.shape[0] - 1, 0))] * inside[..., None]


def _rows(padded, offsets, T):
    """The rows of _padded() in their order."""
    t = torch.arange(T, device=padded.device)
    g = torch.searchsorted(offsets[1:].contiguous(), t.int(), right=True)
    return padded[g, t - offsets[g]]


def _plain_product(s):
    y = torch.bmm(_padded(s["x"], s["offsets"], s["rows_max"]), s["w"].float().transpose(1, 2))
    if s["bias"] is not None:
        y = y + s["bias"][:, None]
    if s["case"]["relu"]:
        y = torch.where(y < 0, 0.0, y)
    return _rows(y, s["offsets"], s["x"].shape[0]).to(DTYPES[s["case"]["out"]])


def _plain_product_dx(s):
    dx = _rows(torch.bmm(_padded(s["dy"], s["offsets"], s["rows_max"]), s["w"].float()), s["offsets"], s["dy"].shape[0])
    if s["h"] is not None:
        dx = dx * (s["h"] > 0)
    return dx.to(DTYPES[s["case"]["out"]])


def _plain_product_dw(s):
    dy = _padded(s["dy"], s["offsets"], s["rows_max"])
    dw = torch.bmm(dy.transpose(1, 2), _padded(s["x"], s["offsets"], s["rows_max"]))
    dw = dw.to(DTYPES[s["case"]["out"]])
    return {"dw": dw, "db": dy.sum(1)} if s["case"]["bias"] else dw


def _plain_logprobs(logits, targets, allowed, temperature, top):
    # a logit at or below -1e30 is a mask's: the lowest value of its type stands for minus infinity
    raw = logits.float()
    raw = torch.where(raw <= -1e30, -math.inf, raw)
    if allowed is not None:
        raw = torch.where(allowed, raw, -math.inf)
    z = raw * (1.0 / temperature)
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    # sum of p z over the entries with p > 0; a row without any has entropy 0
    mean = (torch.where(e > 0, z - m, 0.0) * e).sum(1, keepdim=True)
    entropy = torch.where(total > 0, torch.log(total) - mean / total, 0.0)
    given = z.gather(1, targets.clamp(min=0).long()[:, None])
    logp = torch.where(lse == -math.inf, -math.inf, given - lse)
    out = {"logp": torch.where(targets < 0, 0.0, logp[:, 0]), "entropy": entropy[:, 0], "lse": lse[:, 0]}
    if top:
        # a stable sort: equal logits keep their order, so the lowest index comes first
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :top]
        if order.shape[1] < top:
            order = torch.nn.functional.pad(order, (0, top - order.shape[1]), value=-1)
        best = torch.where(order < 0, -math.inf, z.gather(1, order.clamp(min=0)))
        out["top_logp"] = torch.where(best == -math.inf, -math.inf, best - lse)
        out["top_index"] = torch.where(best == -math.inf, -1, order).to(torch.int32)
    return out


def _plain_logprobs_grad(s):
    c = s["case"]
    z = s["logits"].float() * (1.0 / c["temperature"])
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    if s["allowed"] is not None:
        p, logp = torch.where(s["allowed"], p, 0.0), torch.where(s["allowed"], logp, 0.0)
    dlogp = torch.where(s["targets"] < 0, 0.0, s["dlogp"])
    dz = -p * dlogp[:, None]
    if s["dentropy"] is not None:
        dz = dz - s["dentropy"][:, None] * p * (logp + s["entropy"][:, None])
    at = torch.arange(z.shape[0], device=z.device)
    target = s["targets"].clamp(min=0).long()
    if s["allowed"] is not None:
        dlogp = torch.where(s["allowed"][at, target], dlogp, 0.0)
    dz[at, target] += dlogp
    return (dz * (1.0 / c["temperature"])).to(s["logits"].dtype)


def _to_8(a, seed=None):
    """Values as 8-bit floats (4 exponent, 3 mantissa bits) and one scale for each BLOCK of them,
    rounded to nearest, or up or down at random by `seed`; then what is not 0 stays so."""
    a = a.view(-1, BLOCK)
    most = a.abs().amax(1, keepdim=True)
    most = torch.where(most < 1e-30, 0.0, most)
    x = torch.where(most > 0, a * (448.0 / most), 0.0)
    if seed is not None:
        low = torch.where(x < 2.0 ** -6, 2.0 ** -6, 0.0)      # below, the values are evenly spaced
        bits = (x + low).view(torch.int32) + (_bits(x.numel(), seed, x.device) >> 12).int().view(-1, BLOCK)
        x = torch.where((a > 0) & (most > 0), torch.clamp((bits & ~0xFFFFF).view(torch.float32) - low, min=2.0 ** -9), 0.0)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(-1), (most * (1.0 / 448.0))[:, 0]


def _bits(n, seed, device):
    """32 random bits for each of n places, from the place and the seed alone."""
    x = (torch.arange(n, device=device) + (seed & 0xFFFFFFFF) * 0xBB67AE85) & 0xFFFFFFFF
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 13)


def _from_8(codes, scale):
    return codes.float().view(-1, BLOCK) * scale[:, None]


def _plain_adamw(s):
    s["t"] += 1
    c1, c2 = 1 - BETA1 ** s["t"], math.sqrt(1 - BETA2 ** s["t"])
    shape = (-1, BLOCK)
    g = s["g"].float().view(shape)
    if s["scale"] is not None:
        g = g * s["scale"]
    if s["case"]["bits"] == 32:
        m, v = s["m"].view(shape), s["v"].view(shape)
    else:
        m, v = _from_8(s["m"], s["m_scale"]), _from_8(s["root"], s["root_scale"]).square()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    p = s["p"].view(shape)
    p = p * (1 - s["lr"] * s["decay"]) - (s["lr"] / c1) * (m / (root / c2 + EPS))
    s["p"].copy_(p.view(-1))
    if s["copy"] is not None:
        s["copy"].copy_(s["p"])
    if s["case"]["bits"] == 32:
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
    else:
        s["m"], s["m_scale"] = _to_8(m)
        s["root"], s["root_scale"] = _to_8(root, s["seed"] + s["t"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_scale", "root", "root_scale") if s.get(k) is not None}


# ---------------------------------------------------------------------- one pass
def run(s):
    op, c = s["op"], s["case"]
    if not own:
        if op == "product":
            return _plain_product(s)
        if op == "product_dx":
            return _plain_product_dx(s)
        if op == "product_dw":
            return _plain_product_dw(s)
        if op == "logprobs":
            return _plain_logprobs(s["logits"], s["targets"], s["allowed"], c["temperature"], c["top"])
        if op == "logprobs_grad":
            return _plain_logprobs_grad(s)
        return _plain_adamw(s)
    from paper_1903_05133_gb300 import operators as ops
    if op == "product":
        return ops.grouped_product(s["x"], s["w"], s["offsets"], bias=s["bias"], relu=c["relu"],
                                   out_dtype=DTYPES[c["out"]])
    if op == "product_dx":
        return ops.grouped_product_dx(s["dy"], s["w"], s["offsets"], h=s["h"], out_dtype=DTYPES[c["out"]])
    if op == "product_dw":
        r = ops.grouped_product_dw(s["dy"], s["x"], s["offsets"], bias_grad=c["bias"], out_dtype=DTYPES[c["out"]])
        return {"dw": r[0], "db": r[1]} if c["bias"] else r
    if op == "logprobs":
        r = ops.token_logprobs(s["logits"], s["targets"], top=c["top"], temperature=c["temperature"],
                               allowed=s["allowed"])
        return {k: v for k, v in r._asdict().items() if v is not None}
    if op == "logprobs_grad":
        return ops.token_logprobs_backward(s["logits"], s["targets"], s["lse"], s["entropy"], s["dlogp"],
                                           s["dentropy"], temperature=c["temperature"], allowed=s["allowed"])
    o = s["opt"]
    o.step(s["grads"], lr=s["lr"], grad_scale=s["scale"], seed=s["seed"] + o.t + 1)
    return {k: v for k, v in (("p", s["p"]), ("copy", s["copy"]), *o.state_dict().items())
            if k != "t" and v is not None}


# ---------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("product"):
        return _exact_product(s, case)
    if op.startswith("logprobs"):
        return _exact_logprobs(s, case)
    return _exact_adamw(s, case)


def _exact_product(s, case):
    at = s["offsets"].tolist()
    T, G, K, N = (case[k] for k in ("rows", "groups", "inner", "outer"))
    op = case["op"]
    if op == "product_dw":
        dw = np.zeros((G, N, K))
        db = np.zeros((G, N))
        for g in range(G):
            dy, x = s["dy"][at[g]:at[g + 1]].double(), s["x"][at[g]:at[g + 1]].double()
            dw[g], db[g] = (dy.T @ x).cpu().numpy(), dy.sum(0).cpu().numpy()
        return {"dw": dw, "db": db} if case["bias"] else dw
    out = np.zeros((T, N if op == "product" else K))
    for g in range(G):
        if at[g + 1] == at[g]:
            continue
        w = s["w"][g].double()
        if op == "product":
            y = s["x"][at[g]:at[g + 1]].double() @ w.T
            if s["bias"] is not None:
                y += s["bias"][g].double()
            if case["relu"]:
                y = y.clamp(min=0)
        else:
            y = s["dy"][at[g]:at[g + 1]].double() @ w
            if s["h"] is not None:
                y = y * (s["h"][at[g]:at[g + 1]] > 0)
        out[at[g]:at[g + 1]] = y.cpu().numpy()
    return out


def _exact_logprobs(s, case):
    T, V, top = case["rows"], case["classes"], case.get("top", 0)
    grad = case["op"] == "logprobs_grad"
    r = {k: [] for k in ("logp", "entropy", "lse", "top_logp", "dz")}
    step = max(1, (1 << 26) // V)
    for a in range(0, T, step):
        raw = s["logits"][a:a + step].double()
        ok = torch.ones_like(raw, dtype=torch.bool) if s["allowed"] is None else s["allowed"][a:a + step]
        z = (raw / case["temperature"]).masked_fill(~ok, -math.inf)
        lse = torch.logsumexp(z, 1)
        lp = z - lse[:, None]
        p = torch.where(ok, torch.exp(lp), 0.0)
        lp = torch.where(ok, lp, -math.inf)
        ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
        t = s["targets"][a:a + step].long()
        if grad:
            # d logp_t / d z = onehot - p; d entropy / d z = -p (log p + entropy)
            one = torch.zeros_like(p)
            one[torch.arange(len(t), device=t.device), t.clamp(min=0)] = 1
            d = torch.where(t < 0, 0.0, s["dlogp"][a:a + step].double())
            dz = (one - p) * d[:, None]
            if s["dentropy"] is not None:
                dz = dz - s["dentropy"][a:a + step].double()[:, None] * torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
            r["dz"].append((torch.where(ok, dz, 0.0) / case["temperature"]).cpu().numpy())
            continue
        got = lp.gather(1, t.clamp(min=0)[:, None])[:, 0]
        r["logp"].append(torch.where(t < 0, 0.0, got).cpu().numpy())
        r["entropy"].append(ent.cpu().numpy())
        r["lse"].append(lse.cpu().numpy())
        if top:
            best = torch.sort(lp, dim=1, descending=True).values[:, :top].cpu().numpy()
            r["top_logp"].append(np.pad(best, ((0, 0), (0, top - best.shape[1])), constant_values=-np.inf))
    if grad:
        return np.concatenate(r["dz"])
    out = {k: np.concatenate(r[k]) for k in ("logp", "entropy", "lse")}
    if top:
        out |= {"top_logp": np.concatenate(r["top_logp"]), "top_index": None}
    return out


def _grid():
    """The non-negative values of an 8-bit float with 4 exponent and 3 mantissa bits, in order."""
    low = [k * 2.0 ** -9 for k in range(8)]
    return np.array(low + [(8 + k) / 8 * 2.0 ** e for e in range(-6, 9) for k in range(8)][:-1])


def _exact_adamw(s, case):
    d = lambda a: a.double().cpu().numpy()  # noqa: E731
    n = s["p"].numel()
    if n > 100_000_000:
        return None                          # over 20 seconds on the host
    t = s["t"] + 1
    blocks = lambda a: a.reshape(-1, BLOCK)  # noqa: E731
    g = blocks(d(s["g"]))
    if s["scale"] is not None:
        g = g * d(s["scale"])[0]
    if case["bits"] == 32:
        m, v = blocks(d(s["m"])), blocks(d(s["v"]))
    else:
        m = blocks(d(s["m"])) * d(s["m_scale"])[:, None]
        v = (blocks(d(s["root"])) * d(s["root_scale"])[:, None]) ** 2
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
    lr, p = s["lr"], blocks(d(s["p"]))
    p = p - lr * d(s["decay"]) * p - lr * (m / (1 - BETA1 ** t)) / (np.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"p": p.reshape(-1)}
    if s["copy"] is not None:
        out["copy"] = p.reshape(-1)
    if case["bits"] == 32:
        return out | {"m": m.reshape(-1), "v": v.reshape(-1)}
    grid, root = _grid(), np.sqrt(v)
    for name, a in (("m", m), ("root", root)):
        most = np.abs(a).max(1, keepdims=True)
        most[most < 1e-30] = 0
        x = np.abs(np.divide(a * 448, most, out=np.zeros_like(a), where=most > 0)).clip(max=448).reshape(-1)
        k = np.searchsorted(grid, x, side="right") - 1           # the value at or below
        up = np.minimum(k + 1, len(grid) - 1)
        share = np.where(up > k, (x - grid[k]) / np.where(up > k, grid[up] - grid[k], 1), 0)
        if name == "m":
            at = np.where((share > 0.5) | ((share == 0.5) & (k % 2 == 1)), up, k)
        else:
            j = (np.arange(n, dtype=np.uint64) + np.uint64(((s["seed"] + t) * 0xBB67AE85) & 0xFFFFFFFF)).astype(np.uint32)
            j = (j * np.uint32(0x9E3779B9)).astype(np.uint32)
            j = ((j ^ (j >> np.uint32(15))) * np.uint32(0x6A09E667)).astype(np.uint32)
            j = j ^ (j >> np.uint32(13))
            at = np.where(share + (j >> np.uint32(12)) / 2.0 ** 20 >= 1, up, k)
            at = np.where(x > 0, np.maximum(at, 1), 0)
        out[name] = np.copysign(grid[at], a.reshape(-1))
        out[name + "_scale"] = most[:, 0] / 448
    return out
