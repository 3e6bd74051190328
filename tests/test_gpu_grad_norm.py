"""The norm of all gradients and clipping, on the GPU, against sums in 64 bits."""
import math
import random

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF

pytestmark = pytest.mark.gpu
# squares: 32 one after the other in fp32 and 5 steps of a warp, half of it in the root, two more roundings at the end
TOL = 2.0 ** -24 * 21


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def want_norm(grads, P=None):
    rows = [g.double().reshape(P or 1, -1) for g in grads]
    return torch.cat(rows, 1).square().sum(1).sqrt()


def check(grads, max_norm, learners=None):
    want = want_norm(grads, learners)
    before = [g.clone() for g in grads]
    r = ops.grad_norm(grads, max_norm=max_norm, learners=learners)
    assert r.norm.shape == r.scale.shape == (learners or 1,)
    assert ((r.norm.double() - want).abs() <= TOL * want + 1e-45).all()
    scale = torch.where(want > max_norm, max_norm / want, 1.0)
    assert ((r.scale.double() - scale).abs() <= TOL * scale).all()
    assert ops.grad_norm(grads, learners=learners).scale is None
    assert torch.equal(ops.grad_norm(grads, learners=learners).norm, r.norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    c = ops.clip_gradients(grads, max_norm, learners=learners)
    assert torch.equal(c.norm, r.norm) and torch.equal(c.scale, r.scale)
    for g, b in zip(grads, before):
        s = c.scale.view(-1, *[1] * (g.dim() - 1)) if learners else c.scale.view([])
        assert torch.equal(g, (b.float() * s).to(g.dtype))   # one product, one rounding


@pytest.mark.parametrize("dtype", [F, BF, HF, "mixed"])
@pytest.mark.parametrize("sizes", [[1], [7], [8192], [8193, 1], [3, 0, 100000, 5], [16384 * 3 + 5] * 2, list(range(1, 90)), [33] * 500,
                                   [5] * 3000])
def test_norm(sizes, dtype):
    kinds = [F, BF, HF] if dtype == "mixed" else [dtype]
    at = [(kinds[i % len(kinds)], n) for i, n in enumerate(sizes)]
    for max_norm in (1e-3, 1.0, 1e9):
        grads = [torch.randn(n, generator=gen(i), device="cuda").to(t) for i, (t, n) in enumerate(at)]
        check(grads, max_norm)


@pytest.mark.parametrize("P,shapes", [(1, [(3, 5)]), (4, [(20, 33), (20,)]), (16, [(1,)] * 70), (3, [(130, 129), ()]), (5, [(40000,), (0,), (3,)])])
def test_learners(P, shapes):
    grads = []
    for i, s in enumerate(shapes):
        g = torch.randn(P, *s, generator=gen(i), device="cuda") * torch.arange(P, device="cuda").view(-1, *[1] * len(s))
        grads.append(g.to([F, BF, HF][i % 3]))
    n = sum(math.prod(s) for s in shapes)
    check(grads, 1.5 * math.sqrt(n), learners=P)             # the first one's are zero, some are over it


def test_single_numbers_and_empty_tensors():
    one = torch.tensor(-3.0, device="cuda", dtype=HF)
    none = torch.zeros(0, 4, device="cuda")
    check([one, none, torch.tensor([4.0], device="cuda")], 2.5)
    r = ops.clip_gradients([none, none.clone()], 1.0)
    assert r.norm.item() == 0 and r.scale.item() == 1
    r = ops.grad_norm([torch.zeros(3, 0, device="cuda")], max_norm=1.0, learners=3)
    assert r.norm.tolist() == [0] * 3 and r.scale.tolist() == [1] * 3


def test_the_binding_and_the_host_module_agree():
    s = torch.cuda.current_stream()
    for sizes, P in (([5000] * 3, None), ([64, 130] * 40, 2), ([200000, 3], None)):
        grads = [torch.randn(P or 1, n, generator=gen(n), device="cuda").to([F, BF][i % 2]) for i, n in enumerate(sizes)]
        a, b = ops.grad_norm(grads, 1.0, P), ops.grad_norm(grads, 1.0, P, stream=s)
        assert torch.equal(a.norm, b.norm) and torch.equal(a.scale, b.scale)
        other = [g.clone() for g in grads]
        ops.clip_gradients(grads, 1.0, P), ops.clip_gradients(other, 1.0, P, stream=s)
        assert all(torch.equal(x, y) for x, y in zip(grads, other))


def test_one_buffer_of_odd_sizes():
    r = random.Random(4)
    for dtype in (F, BF, HF):
        sizes = [r.randint(1, 20000) for _ in range(400)]
        flat = torch.randn(sum(sizes) + 1, generator=gen(1), device="cuda").to(dtype)
        grads, at = [], 1
        for n in sizes:
            grads.append(flat[at:at + n])
            at += n
        first = flat[0].clone()
        check(grads, 5.0)
        check(grads[::-1], 2.0)
        assert flat[0] == first


def test_squares_beyond_fp32():
    for dtype, values in ((F, (1e-30, 1e-44, 1e25, 3e38)), (BF, (1e-30, 1e-38, 1e25, 3e38)), (HF, (6e-8, 65504.0))):
        for v in values:
            g = torch.full((50000,), v, device="cuda").to(dtype)
            g[1::2] *= -1
            want = want_norm([g])
            got = ops.grad_norm([g], max_norm=1.0)
            if want > torch.finfo(F).max:                    # no fp32 number
                assert got.norm.item() == math.inf
            else:
                # a norm of 1e-44 * sqrt(50000) = 2.2e-42 is a multiple of 2^-149 when rounded: half of that
                assert abs(got.norm.double() - want) <= TOL * want + 2.0 ** -150
            assert abs(got.scale.double() - min(1.0, 1.0 / want.item())) <= TOL
    # small ones beside large ones, and zeros
    g = torch.cat([torch.full((9000,), 1e-25, device="cuda"), torch.zeros(40000, device="cuda"), -torch.zeros(9000, device="cuda")])
    check([g, torch.full((100,), 1e-24, device="cuda")], 1e-24)
    z = torch.zeros(20000, device="cuda", dtype=BF)
    r = ops.clip_gradients([z, -z], 0.0)
    assert r.norm.item() == 0 and r.scale.item() == 1
    # a norm that fp32 does not hold, infinities and NaN
    big = torch.full((1 << 16,), 3e38, device="cuda")
    r = ops.grad_norm([big], max_norm=1e38)
    assert r.norm.item() == math.inf and abs(r.scale.item() / (1e38 / (3e38 * 256)) - 1) < 1e-6
    g = torch.ones(30000, device="cuda")
    g[29999] = math.inf
    r = ops.grad_norm([g, g.clone()], max_norm=1.0)
    assert r.norm.item() == math.inf and r.scale.item() == 0
    g[5] = math.nan
    r = ops.clip_gradients([g], 1.0)
    assert r.norm.isnan().all() and r.scale.item() == 1 and g[0] == 1


def test_zero_largest_norm_and_the_same_tensor_twice():
    g = torch.ones(100, device="cuda")
    assert ops.grad_norm([g, g], max_norm=1.0).norm.item() == pytest.approx(math.sqrt(200), rel=1e-6)
    flat = torch.ones(1000, device="cuda")
    for bad in ([g, g], [flat[:600], flat[599:]], [flat[500:], g, flat[:501]]):
        with pytest.raises(ValueError, match="share memory"):
            ops.clip_gradients(bad, 1.0)
    assert (flat == 1).all()
    r = ops.clip_gradients([g], 0.0)
    assert r.scale.item() == 0 and (g == 0).all()


def test_with_adamw():
    # grad_scale takes the factor, which is the same step as clipping first
    make = lambda: [torch.ones(300, device="cuda"), torch.ones(41, 7, device="cuda")]  # noqa: E731
    grads = [torch.randn(300, generator=gen(0), device="cuda"), torch.randn(41, 7, generator=gen(1), device="cuda")]
    a, b = make(), make()
    oa, ob = ops.AdamW(a), ops.AdamW(b)
    oa.step(grads, lr=0.1, grad_scale=ops.grad_norm(grads, max_norm=0.5).scale)
    ops.clip_gradients(grads, 0.5)
    ob.step(grads, lr=0.1)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(oa.m, ob.m)


def test_captured_and_on_a_stream():
    grads = [torch.randn(40001, generator=gen(0), device="cuda"), torch.randn(77, generator=gen(1), device="cuda").to(BF)]
    start = [g.clone() for g in grads]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = ops.grad_norm(grads, max_norm=1.0, stream=s)
    s.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            got.append(ops.clip_gradients(grads, 1.0))
    for graph, r in zip(graphs, got):
        for g, b in zip(grads, start):
            g.copy_(b)
        graph.replay()
        assert torch.equal(r.norm, want.norm) and torch.equal(r.scale, want.scale)
        assert torch.equal(grads[0], start[0] * want.scale)


def test_local_adamw_clips_each_learner():
    # the first moments of a first step are 0.1 of the gradients: with a norm given each learner's are scaled by its factor
    from paper_1903_05133_gb300.inputs import learner_data, perturbed_layers
    from paper_1903_05133_gb300.local_adamw import LocalAdamW, ragged_batches
    from test_gpu_local_adamw import W
    X, y = learner_data(W, device="cuda")
    x, t, off = next(ragged_batches(X, y, W.B, 5))
    models = {}
    for max_norm in (None, 1e9, 0.5):
        m = models[max_norm] = LocalAdamW(W.P, W.S, W.K1, W.K2, W.lr, W.dims, bits=32, max_norm=max_norm)
        m.load(perturbed_layers(W, 0.01, seed=3))
        m.step(x, t, off)

    def moments(m):
        # [P] rows of every tensor's first moments, which stand from multiples of 256 on
        rows = []
        for opt, tensors in ((m.opt_w, [w for w, _ in m.layers]), (m.opt_b, [b for _, b in m.layers])):
            at = 0
            for v in tensors:
                n = v[0].numel()
                rows.append(torch.stack([opt.m[at + j * -(-n // 256) * 256:][:n] for j in range(W.P)]))
                at += W.P * -(-n // 256) * 256
        return torch.cat(rows, 1).double()
    free, loose, tight = (moments(models[n]) for n in (None, 1e9, 0.5))
    assert torch.equal(free, loose)
    norms = 10 * free.norm(dim=1)
    assert (norms > 0.5).any()
    scale = torch.where(norms > 0.5, 0.5 / norms, 1.0)
    # the weights' gradients are rounded to bf16 once more
    assert (tight - free * scale[:, None]).norm() <= 2.0 ** -8 * tight.norm()
    assert ((10 * tight.norm(dim=1) - torch.minimum(norms, torch.full_like(norms, 0.5))).abs() <= 2.0 ** -8 * norms).all()
