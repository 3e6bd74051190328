"""The router, the sort by group and the rows' way to their groups and back, on the GPU, against the formulas
in 64 bits."""
import math

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF, U

pytestmark = pytest.mark.gpu
TYPES = [F, BF, HF]
LOWEST = {t: torch.finfo(t).min for t in TYPES}


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def want_sort(group, G):
    g = group.cpu().reshape(-1).long()
    key = torch.where((g >= 0) & (g < G), g, G)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(len(order))
    n = int((key < G).sum())
    offsets = torch.searchsorted(key[order], torch.arange(G + 1))
    source = torch.where(torch.arange(len(order)) < n, order, -1)
    return offsets, torch.where(key < G, place, -1).view(group.shape), source


def check_sorted(r, group, G):
    for got, want in zip((r.offsets, r.place, r.source), want_sort(group, G)):
        assert got.dtype == torch.int32 and torch.equal(got.cpu().long(), want)


def want_route(z, k, over):
    """On the CPU: experts, weights, lse, and the distance of the chosen logits to the largest."""
    z = z.double().cpu()
    bad = ~(z < math.inf).all(1)
    z = torch.where(z <= -1e30, -math.inf, z)
    best, e = torch.sort(z, dim=1, descending=True, stable=True)
    best, e = best[:, :k], e[:, :k]
    m = torch.where(best[:, :1].isinf(), 0.0, best[:, :1])
    total = torch.exp(z - m).sum(1, keepdim=True)
    x = torch.exp(best - m)
    w = x / (x.sum(1, keepdim=True) if over == "chosen" else total)
    none = best == -math.inf
    w = torch.where(none, 0.0, w)
    lse = (m + total.log())[:, 0]
    w[bad] = math.nan
    lse[bad] = math.nan
    return torch.where(none | bad[:, None], -1, e), w, lse, torch.where(none, 0.0, m - best)


def check_route(z, k, over, learners=None):
    r = ops.route(z, k, over=over, learners=learners)
    e, w, lse, d = want_route(z, k, over)
    assert torch.equal(r.experts.cpu().long(), e)
    # each exponential: its argument's rounding and 2^-22 of the hardware's; their sum has the largest's weight
    tol = 2.0 ** -22 * (16 + d) * w
    got = r.weights.cpu().double()
    assert torch.equal(got.isnan(), w.isnan()) and ((got - w).abs() <= tol + 1e-38)[~w.isnan()].all()
    got, fin = r.lse.cpu().double(), lse.isfinite()
    assert torch.equal(got.isnan(), lse.isnan()) and torch.equal(got == -math.inf, lse == -math.inf)
    assert ((got - lse).abs() <= 2.0 ** -22 * (16 + lse.abs()))[fin].all()
    E = z.shape[1]
    group, G = e, E
    if learners is not None:
        at = learners.cpu().long()
        t = torch.arange(z.shape[0])
        p = torch.searchsorted(at[1:].contiguous(), t, right=True)
        P = len(at) - 1
        p = torch.where((t < at[0]) | (p >= P), -1, p)
        group = torch.where((e < 0) | (p[:, None] < 0), -1, e + p[:, None] * E)
        G = P * E
    check_sorted(r, group, G)
    return r


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("over", ["chosen", "all"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (8, 64, 6), (3, 33, 33 - 1), (33, 5, 5), (256, 60, 8), (257, 60, 8),
                                   (700, 128, 8), (1000, 200, 3), (513, 513, 4), (40, 1024, 32), (2500, 1024, 16),
                                   (20001, 4, 1), (6000, 7, 7)])
def test_route(T, E, k, over, dtype):
    z = torch.randn(T, E, generator=gen(T + E), device="cuda").to(dtype)
    check_route(z, k, over)
    # equal logits
    check_route(torch.randint(-2, 3, (T, E), generator=gen(T), device="cuda").to(dtype), k, over)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(9, 40, 5), (500, 130, 8), (1200, 600, 4)])
def test_route_masks(T, E, k, dtype):
    g = gen(E)
    z = torch.randn(T, E, generator=g, device="cuda")
    out = torch.rand(T, E, generator=g, device="cuda") < 0.9
    out[0] = True                                            # nothing is left
    out[1] = True
    out[1, E - 1] = False                                    # one
    for low in (-math.inf, LOWEST[dtype]):
        if dtype == HF and low != -math.inf:
            continue                                         # fp16's lowest is a number like others
        check_route(z.to(dtype).masked_fill(out, low), k, "chosen")
        check_route(z.to(dtype).masked_fill(out, low), k, "all")
    z = z.to(dtype)
    z[2, 3], z[3, 0], z[4, E - 1] = math.nan, math.inf, -0.0
    z[5] = 0.0
    z[5, ::2] = -0.0                                         # zeros of both signs are equal
    r = check_route(z, k, "all")
    assert r.experts[5].tolist() == list(range(k)) and (r.experts[2:4] == -1).all()


@pytest.mark.parametrize("T,P,E,k", [(50, 3, 7, 2), (3000, 16, 60, 4), (900, 1, 64, 8), (5000, 128, 8, 2), (4000, 1000, 1, 1)])
def test_route_learners(T, P, E, k):
    z = torch.randn(T, E, generator=gen(T), device="cuda")
    cut = torch.sort(torch.randint(0, T + 1, (P + 1,), generator=gen(P), device="cuda")).values
    check_route(z, k, "chosen", cut.int())                   # rows of no learner, before and behind them
    cut[0], cut[-1] = 0, T
    cut[1] = 0                                               # a learner without rows
    if P > 1:
        check_route(z, k, "chosen", cut.int())
    check_route(z, k, "chosen", torch.full((P + 1,), T, dtype=torch.int32, device="cuda"))


def test_route_strided_and_empty():
    wide = torch.randn(300, 90, generator=gen(1), device="cuda")
    for z in (wide[:, 3:67], wide[::2, :50], wide[:1, 5:20], wide[:, 1:2]):
        check_route(z, min(4, z.shape[1]), "chosen")
    r = ops.route(wide[:0], 3)
    assert r.experts.shape == (0, 3) and r.source.shape == (0,) and r.offsets.tolist() == [0] * 91
    s = ops.sort_by_group(torch.zeros(0, 2, dtype=torch.int32, device="cuda"), 5)
    assert s.offsets.tolist() == [0] * 6


@pytest.mark.parametrize("T,k,G", [(1, 1, 1), (1, 32, 3), (64, 32, 1000), (100, 3, 7), (2049, 1, 2), (300, 8, 64), (70000, 1, 1024),
                                   (200000, 8, 33)])
def test_sort_by_group(T, k, G):
    g = gen(T)
    ids = torch.randint(-1, G + 1, (T, k), generator=g, device="cuda", dtype=torch.int32)      # equal ones in a row, and none
    check_sorted(ops.sort_by_group(ids, G), ids, G)
    same = torch.full((T, k), G - 1, dtype=torch.int32, device="cuda")
    check_sorted(ops.sort_by_group(same, G), same, G)
    none = torch.full((T, k), -2 ** 31, dtype=torch.int32, device="cuda")
    check_sorted(ops.sort_by_group(none, G), none, G)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("over", ["chosen", "all"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 8, 2), (37, 60, 4), (2000, 33, 8), (300, 1024, 32)])
def test_route_backward(T, E, k, over, dtype):
    g = gen(T * E + k)
    z = torch.randn(T, E, generator=g, device="cuda")
    if E > 4:
        z[0, 1:] = -math.inf                                 # fewer experts than k
        z[T - 1, E // 2:] = LOWEST[dtype] if dtype != HF else -math.inf
    z = z.to(dtype)
    dw = torch.randn(T, k, generator=g, device="cuda")
    r = ops.route(z, k, over=over)
    got = ops.route_backward(dw, z, r.experts, r.weights, lse=r.lse, over=over)
    assert got.dtype == dtype
    x = torch.where(z.double() <= -1e30, -math.inf, z.double()).requires_grad_()
    has = r.experts >= 0
    at = r.experts.clamp(min=0).long()
    p = torch.softmax(x, 1)
    w = p.gather(1, at) * has
    if over == "chosen":
        w = w / w.sum(1, keepdim=True)
    (w * dw).sum().backward()
    size = (w.detach() * dw).abs().sum(1, keepdim=True)
    # the probabilities' errors (2^-22 and the arguments' roundings) times the sum, sums of k terms, the result's rounding
    p = p.detach()
    one = torch.zeros_like(p).scatter_(1, at, (w.detach() * dw.abs() * has))
    tol = 2.0 ** -22 * (16 + z.double().abs().clamp(max=100)) * (torch.where(one > 0, 1.0, p) * size + one)
    tol = tol + U[dtype] * x.grad.abs() + (2.0 ** -25 if dtype == HF else 1e-38)
    assert ((got.double() - x.grad).abs() <= tol).all()
    assert (got[z.double() <= -1e30] == 0).all()
    # onto the logits themselves
    same = z.clone()
    assert ops.route_backward(dw, same, r.experts, r.weights, lse=r.lse, over=over, out=same) is same
    assert torch.equal(same, got)


def test_route_backward_rows_without_an_expert_and_bad_ones():
    z = torch.randn(6, 10, generator=gen(3), device="cuda")
    z[1], z[2, 4], z[3, 0] = -math.inf, math.nan, math.inf
    dw = torch.randn(6, 3, generator=gen(4), device="cuda")
    for over in ("chosen", "all"):
        r = ops.route(z, 3, over=over)
        g = ops.route_backward(dw, z, r.experts, r.weights, lse=r.lse, over=over)
        assert (g[1] == 0).all() and g[2:4].isnan().all() and g[[0, 4, 5]].isfinite().all()
    # an expert that is named twice has both entries' gradients
    e = torch.tensor([[2, 2, 5]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.25, 0.5, 0.25]], device="cuda")
    g = ops.route_backward(torch.tensor([[1.0, 2.0, 4.0]], device="cuda"), z[:1], e, w)
    s = 0.25 + 1.0 + 1.0
    assert g[0, 2].item() == 0.25 + 1.0 - 0.75 * s and g[0, 5].item() == 1.0 - 0.25 * s and g[0].count_nonzero() == 2


def test_route_gradient_against_differences():
    z = torch.randn(4, 12, generator=gen(8), device="cuda")
    dw = torch.randn(4, 3, generator=gen(9), device="cuda")
    for over in ("chosen", "all"):
        r = ops.route(z, 3, over=over)
        g = ops.route_backward(dw, z, r.experts, r.weights, lse=r.lse, over=over)
        for t, i in ((0, r.experts[0, 0]), (1, r.experts[1, 2]), (2, z[2].argmin()), (3, r.experts[3, 1])):
            h, up, down = 2.0 ** -8, z.clone(), z.clone()
            up[t, i] += h
            down[t, i] -= h
            loss = lambda v: (ops.route(v, 3, over=over).weights.double() * dw).sum()  # noqa: E731
            # second-order: h^2 times third derivatives below 4 |dw|; 2^-21 of the weights over 2 h
            assert abs((loss(up) - loss(down)) / (2 * h) - g[t, i]) <= 4 * h * h * dw[t].abs().sum() + 2.0 ** -13


# ---------------------------------------------------------------------- rows
def places(T, k, G, seed, dropped=0.2):
    g = gen(seed)
    ids = torch.randint(0, G, (T, k), generator=g, device="cuda", dtype=torch.int32)
    ids = torch.where(torch.rand(T, k, generator=g, device="cuda") < dropped, -1, ids)
    return ops.sort_by_group(ids, G)


WIDTHS = [(1, 1, 1), (5, 2, 7), (3, 8, 8), (30, 3, 64), (9, 1, 100), (64, 4, 257), (17, 6, 1111), (13, 9, 1024), (7, 32, 40),
          (5, 2, 4096), (3, 8, 8195), (1, 2, 20000), (2000, 2, 24)]


def sliced(T, D, dtype, seed, how):
    """Rows with strides: 'even' (contiguous), 'odd' (from an odd column on), 'apart' (aligned, with a gap)."""
    if how == "even":
        return torch.randn(T, D, generator=gen(seed), device="cuda").to(dtype)
    pad, at = (3, 1) if how == "odd" else (16 + -D % 16, 0)
    return torch.randn(T, D + pad, generator=gen(seed), device="cuda").to(dtype)[:, at:at + D]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["even", "odd", "apart"])
@pytest.mark.parametrize("T,k,D", WIDTHS)
def test_dispatch_and_back(T, k, D, how, dtype):
    s = places(T, k, 5, T + D)
    x = sliced(T, D, dtype, 1, how)
    n = int(s.offsets[-1])
    src = s.source[:n].long()
    want = torch.zeros(T * k, D, dtype=dtype, device="cuda")
    want[:n] = x[src // k]
    assert torch.equal(ops.dispatch(x, s.place, s.offsets), want)
    room = torch.full((T * k, D + 9), 7.0, dtype=dtype, device="cuda")
    out = room[:, 2:2 + D]
    assert ops.dispatch(x, s.place, s.offsets, out=out) is out and torch.equal(out, want)
    assert (room[:, :2] == 7).all() and (room[:, 2 + D:] == 7).all()
    # its gradient: a sum of the entries' rows, k roundings in fp32 and the result's
    dxs = sliced(T * k, D, dtype, 2, how)
    for d in {dtype, F}:
        got = ops.dispatch_backward(dxs, s.place, out_dtype=d)
        ref = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, src // k, dxs[:n].double())
        size = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, src // k, dxs[:n].double().abs())
        assert got.dtype == d and ((got.double() - ref).abs() <= k * 2.0 ** -24 * size + U[d] * ref.abs()).all()
    out = torch.full((T, D + 9), 7.0, dtype=dtype, device="cuda")[:, 2:2 + D]
    assert torch.equal(ops.dispatch_backward(dxs, s.place, out=out), ops.dispatch_backward(dxs, s.place))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["even", "odd", "apart"])
@pytest.mark.parametrize("T,k,D", WIDTHS)
def test_combine(T, k, D, how, dtype):
    s = places(T, k, 5, T * D)
    n = int(s.offsets[-1])
    src = s.source[:n].long()
    y = sliced(T * k, D, dtype, 3, how)
    y[n:] = math.nan                                         # rows of no entry are not read
    w = torch.rand(T, k, generator=gen(4), device="cuda")
    terms = y[:n].double() * w.view(-1)[src].double()[:, None]
    ref = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, src // k, terms)
    size = torch.zeros(T, D, dtype=torch.float64, device="cuda").index_add_(0, src // k, terms.abs())
    for d in {dtype, F}:
        got = ops.combine(y, s.place, w, out_dtype=d)
        tiny = 2.0 ** -25 if d == HF else 0.0
        assert got.dtype == d and ((got.double() - ref).abs() <= k * 2.0 ** -24 * size + U[d] * ref.abs() + tiny).all()
        dout = sliced(T, D, d, 5, how)
        dy, dw = ops.combine_backward(dout, y, s.place, w, s.offsets)
        want = dout.float()[src // k] * w.view(-1)[src][:, None]         # one rounding to fp32, then one to the type
        assert torch.equal(dy[:n], want.to(dtype)) and (dy[n:] == 0).all()
        dot = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        mag = dot.clone()
        prod = dout.double()[src // k] * y[:n].double()
        dot[src], mag[src] = prod.sum(1), prod.abs().sum(1)
        # a thread's share one after the other, at most D / 32 of it, then lanes and warps
        off = lambda v: (v.view(-1).double() - dot).abs()  # noqa: E731
        assert (off(dw) <= 2.0 ** -24 * (D / 32 + 24) * mag).all()
    room = torch.full((T * k, D + 9), 7.0, dtype=dtype, device="cuda")
    out = room[:, 2:2 + D]
    dy2, dw2 = ops.combine_backward(dout, y, s.place, w, s.offsets, out=out)
    # the sums' order goes by the rows' alignment
    assert dy2 is out and torch.equal(dy2, dy) and (off(dw2) <= 2.0 ** -24 * (D / 32 + 24) * mag).all()
    assert (room[:, :2] == 7).all() and (room[:, 2 + D:] == 7).all()


def test_rows_without_entries():
    place = torch.full((4, 3), -1, dtype=torch.int32, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    x, y, w = torch.ones(4, 40, device="cuda"), torch.ones(12, 40, device="cuda"), torch.ones(4, 3, device="cuda")
    assert (ops.dispatch(x, place, off) == 0).all() and (ops.combine(y, place, w) == 0).all()
    dy, dw = ops.combine_backward(x, y, place, w, off)
    assert (dy == 0).all() and (dw == 0).all()
    # places that no row has are nowhere
    far = torch.tensor([[12, 2 ** 31 - 1, -2 ** 31]] * 4, dtype=torch.int32, device="cuda")
    assert (ops.combine(y, far, w) == 0).all() and (ops.dispatch(x, far, off) == 0).all()
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    assert ops.dispatch(x[:0], none, off).shape == (0, 40) and ops.combine(y[:0], none, w[:0, :2]).shape == (0, 40)
    assert ops.combine_backward(x[:0], y[:0], none, w[:0, :2], off)[0].shape == (0, 40)


# ---------------------------------------------------------------------- together
def experts_pass(x, router, w1, w2, dout, k, over):
    """Rows through their experts, two layers each, and all gradients."""
    logits = (x.float() @ router.T.float())
    r = ops.route(logits, k, over=over)
    xs = ops.dispatch(x, r.place, r.offsets)
    h = ops.grouped_product(xs, w1, r.offsets, relu=True)
    y = ops.grouped_product(h, w2, r.offsets)
    out = ops.combine(y, r.place, r.weights, out_dtype=F)
    dy, dweights = ops.combine_backward(dout, y, r.place, r.weights, r.offsets)
    dw2 = ops.grouped_product_dw(dy, h, r.offsets, out_dtype=F)
    dh = ops.grouped_product_dx(dy, w2, r.offsets, h=h)
    dw1 = ops.grouped_product_dw(dh, xs, r.offsets, out_dtype=F)
    dxs = ops.grouped_product_dx(dh, w1, r.offsets)
    dx = ops.dispatch_backward(dxs, r.place, out_dtype=F)
    dlogits = ops.route_backward(dweights, logits, r.experts, r.weights, lse=r.lse, over=over)
    return out, dx, dw1, dw2, dlogits, r


def experts_reference(x, router, w1, w2, dout, r, over):
    x, w1, w2 = (v.double().requires_grad_() for v in (x, w1, w2))
    logits = (x.detach().float() @ router.T.float()).double().requires_grad_()
    p = torch.softmax(logits, 1).gather(1, r.experts.long())
    p = p / p.sum(1, keepdim=True) if over == "chosen" else p
    out = 0
    for j in range(r.experts.shape[1]):
        e = r.experts[:, j].long()
        h = torch.relu(torch.bmm(w1[e], x[:, :, None]))
        out = out + p[:, j, None] * torch.bmm(w2[e], h)[:, :, 0]
    (out * dout.double()).sum().backward()
    return out, x.grad, w1.grad, w2.grad, logits.grad


@pytest.mark.parametrize("over", ["chosen", "all"])
@pytest.mark.parametrize("T,E,k,D,H", [(70, 8, 2, 64, 96), (9, 5, 3, 40, 24), (600, 16, 4, 128, 64)])
def test_a_layer_of_experts(T, E, k, D, H, over):
    g = gen(T)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, router = n(T, D).to(BF), n(E, D) / math.sqrt(D)
    w1, w2 = (n(E, H, D) / math.sqrt(D)).to(BF), (n(E, D, H) / math.sqrt(H)).to(BF)
    dout = n(T, D)
    *got, r = experts_pass(x, router, w1, w2, dout, k, over)
    want = experts_reference(x, router, w1, w2, dout, r, over)
    for a, b in zip(got, want):
        # rows pass through bf16 four times at most (2^-9 of each on average; 2^-8 at worst)
        assert (a.double() - b).norm() <= 4 * 2.0 ** -8 * b.norm()
    ops.operator_check()


def test_captured_and_replayed():
    T, E, k, D, H = 300, 8, 2, 64, 96
    g = gen(7)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, router, dout = n(T, D).to(BF), n(E, D), n(T, D)
    w1, w2 = n(E, H, D).to(BF), n(E, D, H).to(BF)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        experts_pass(x, router, w1, w2, dout, k, "chosen")
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(experts_pass(x, router, w1, w2, dout, k, "chosen"))
    for seed in (1, 2, 3):
        x.copy_(torch.randn(T, D, generator=gen(seed), device="cuda"))
        for graph in graphs:
            graph.replay()
        want = experts_pass(x, router, w1, w2, dout, k, "chosen")
        for got in outs:
            for a, b in zip(got[:-1], want[:-1]):
                assert torch.equal(a, b)
            for a, b in zip(got[-1], want[-1]):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    T, E, k, D = 4000, 64, 4, 256
    z = torch.randn(T, E, generator=gen(1), device="cuda")
    x = torch.randn(T, D, generator=gen(2), device="cuda").to(BF)
    want = ops.route(z, k)
    xs = ops.dispatch(x, want.place, want.offsets)
    out = ops.combine(xs, want.place, want.weights)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(20):
        for s in streams:
            r = ops.route(z, k, stream=s)
            a = ops.dispatch(x, r.place, r.offsets, stream=s)
            got.append((r, a, ops.combine(a, r.place, r.weights, stream=s)))
    torch.cuda.synchronize()
    for r, a, b in got:
        assert all(torch.equal(p, q) for p, q in zip(r, want)) and torch.equal(a, xs) and torch.equal(b, out)


def test_the_binding_and_the_host_module_agree():
    s = torch.cuda.current_stream()
    for T, E, k, D in ((5, 8, 2, 40), (700, 60, 4, 129), (3000, 256, 8, 256)):
        z = torch.randn(T, E, generator=gen(T), device="cuda").to(BF)
        cut = torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")
        learners = cut if 2 * E <= 1024 else None
        a, b = ops.route(z, k, "all", learners), ops.route(z, k, "all", learners, stream=s)
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        x = torch.randn(T, D, generator=gen(D), device="cuda").to(BF)
        xs = ops.dispatch(x, a.place, a.offsets)
        assert torch.equal(xs, ops.dispatch(x, a.place, a.offsets, stream=s))
        for d in (None, F):
            assert torch.equal(ops.combine(xs, a.place, a.weights, out_dtype=d), ops.combine(xs, a.place, a.weights, out_dtype=d, stream=s))
            assert torch.equal(ops.dispatch_backward(xs, a.place, out_dtype=d), ops.dispatch_backward(xs, a.place, out_dtype=d, stream=s))
        p, q = ops.combine_backward(x, xs, a.place, a.weights, a.offsets), ops.combine_backward(x, xs, a.place, a.weights, a.offsets, stream=s)
        assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])
        for over in ("chosen", "all"):
            assert torch.equal(ops.route_backward(p[1], z, a.experts, a.weights, a.lse, over),
                               ops.route_backward(p[1], z, a.experts, a.weights, a.lse, over, stream=s))


def test_many_equal_logits_of_large_routers():
    # fp32 logits of which many are equal, at widths of every kernel, with more chosen than different values
    for T, E, k in ((50, 16, 16), (200, 64, 8), (100, 100, 8), (64, 128, 16), (70, 250, 12), (40, 128, 32), (40, 500, 20), (40, 1000, 32)):
        g = gen(E)
        z = torch.randint(0, 3, (T, E), generator=g, device="cuda").float()
        z[::4] = 1.0
        z[1::4, E // 2:] = -math.inf
        z[2::4] = torch.randn(len(z[2::4]), E, generator=g, device="cuda")         # rows without, beside those
        check_route(z, k, "chosen")
        check_route(z, k, "all")
