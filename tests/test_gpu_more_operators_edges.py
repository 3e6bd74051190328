"""Where the routing, row, norm and draft operators can go wrong: noise and masks at the ends of their ranges, results
that are kept, values that must not vanish."""
import math

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF
from test_gpu_verify_drafts import check, gen, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


# Sequences and classes of one kernel, of two, and of two with many CTAs a sequence.
SIZES = [(6, 2), (6, 300), (600, 50), (3, 40001)]


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("B,V", SIZES)
def test_noise_of_any_size(B, V, dtype):
    # a class of p = 1 beside one of p = 1e-6, both with noise whose reciprocal is below the normal range of fp32
    z = torch.full((B, 1, V), -math.inf, device="cuda")
    z[:, 0, 0], z[:, 0, V - 1] = 0.0, -13.8
    none = torch.zeros(B, 0, device="cuda")
    noise = torch.ones(B, V, device="cuda")
    noise[:, 0], noise[:, V - 1] = 1e38, 8e37
    r = check(z.to(dtype), none.int(), none, noise)
    assert (r.tokens == 0).all()
    # scores over the whole range of positive fp32 numbers, and beyond where they are the largest
    g = gen(V)
    for low, high in ((-149, 127), (100, 127), (126, 127.99), (-149, -120)):
        power = torch.rand(B, V, generator=g, device="cuda", dtype=torch.float64) * (high - low) + low
        noise = (2.0 ** power).float()
        for probs, masked in ((F, True), (None, False)):
            z, x, u, _, q, ok = make(B, 1, V, dtype, probs, masked, 1.0, V, sure=False)
            check(z * 4, x, u, noise, q, ok)
            check(z * 4, x, torch.ones_like(u), noise, q, ok)


@pytest.mark.parametrize("B,V", SIZES)
def test_noise_next_to_the_largest_number(B, V):
    # all scores are subnormal: neighbours are told apart all the same
    g = gen(V)
    most = torch.finfo(F).max
    noise = most * (1 - torch.rand(B, V, generator=g, device="cuda") * 1e-3)
    none = torch.zeros(B, 0, device="cuda")
    check(torch.randn(B, 1, V, generator=g, device="cuda") * 1e-3, none.int(), none, noise)
    check(torch.zeros(B, 1, V, device="cuda"), none.int(), none, torch.full((B, V), most, device="cuda"))


@pytest.mark.parametrize("above", [20.0, 60.0, 200.0])
@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("B,V", [(6, 40), (600, 40), (6, 20011)])
def test_the_only_class_rejected_beside_masked_ones_far_above_it(B, V, dtype, above):
    # nothing is left of p but the draft itself; the masked logits say nothing, however large they are
    g = gen(V)
    z = (torch.randn(B, 2, V, generator=g, device="cuda") + above).to(dtype)
    z[:, :, 5] = 0.0
    ok = torch.zeros(V, dtype=torch.bool, device="cuda")
    ok[5] = True
    x = torch.full((B, 1), 5, dtype=torch.int32, device="cuda")
    u = torch.ones(B, 1, device="cuda")                      # not below p = 1
    noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    r = check(z, x, u, noise, None, ok.expand(B, 2, V))
    assert (r.tokens[:, 0] == 5).all() and (r.logp[:, 0] == 0).all()
    # and where the draft is the largest but one of two allowed
    ok[7] = True
    z[:, :, 7] = -9.0
    r = check(z, x, u, noise, None, ok.expand(B, 2, V))
    assert (r.tokens[:, 0] == 7).all()


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("B,V", [(8, 3), (8, 333), (600, 70), (4, 40001)])
def test_logits_next_to_a_masks_at_the_highest_temperature(B, V, dtype):
    # -1e30 is a mask's even where 1e27 apart is a factor e
    g = gen(V)
    z = -9.9e29 - 9.9e27 * torch.rand(B, 3, V, generator=g, device="cuda")
    z[torch.rand(B, 3, V, generator=g, device="cuda") < 0.7] = -1.0025e30 if dtype == BF else -1e30
    z[torch.rand(B, 3, V, generator=g, device="cuda") < 0.1] = -math.inf
    z[:, :, V // 2] = -9.97e29
    z = z.to(dtype)
    assert (z.double()[:, :, V // 2] > -1e30).all()
    x = torch.full((B, 2), V // 2, dtype=torch.int32, device="cuda")
    noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    u = torch.rand(B, 2, generator=g, device="cuda") * 0.01
    check(z, x, u, noise, None, None, 1e27)
    check(z, x, torch.ones_like(u), noise, None, None, 1e27)
    q = torch.full((B, 2, V), 0.5 / V, device="cuda")
    check(z, x, torch.ones_like(u), noise, q, None, 1e27)
    ok = torch.rand(V, generator=g, device="cuda") < 0.8
    ok[V // 2] = True
    check(z, x, u, noise, None, ok.expand(B, 3, V), 1e27)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V,B", [(128000, 1300), (5000, 700), (2001, 500)])
def test_logits_that_rise_along_the_row(V, B, dtype):
    # each batch of a thread has a new largest logit, and the sum is rescaled; u is next to p, a step of 2^-26 to 2^-14 away
    g = gen(V)
    for step in (1e-5, 3e-4) if dtype == F else (2e-4,):
        row = (torch.arange(V, device="cuda") * step).to(dtype)
        z = row.expand(B, 2, V)
        lp = torch.log_softmax(row.double(), 0)
        x = V - 1 - torch.randint(0, 50, (B, 1), generator=g, device="cuda")
        p = torch.exp(lp[x])
        away = 2.0 ** (-26 + 12 * torch.rand(B, 1, generator=g, device="cuda", dtype=torch.float64))
        sign = torch.randint(0, 2, (B, 1), generator=g, device="cuda") * 2 - 1
        u = (p * (1 + sign * away)).float()
        noise = torch.ones(1, V, device="cuda").expand(B, V)
        r = ops.verify_drafts(z, x, u, noise)
        # the two sides are exact numbers but for 2^-45
        sure = (u.double() - p).abs() > 2.0 ** -40 * p
        want = u.double() < p
        assert torch.equal((r.accepted == 1)[:, None][sure], want[sure])


@pytest.mark.parametrize("temperature", [1.0, 0.7, 1.3, 0.37])
@pytest.mark.parametrize("B,V", [(40, 700), (600, 300), (40, 30011)])
def test_log_probabilities_are_rounded_once(B, V, temperature):
    # V - 1 equal classes, whose sum is exact, and the draft's below them by a distance at which the sum does not see it
    g = gen(V)
    z = torch.full((B, 2, V), 3.25, device="cuda")
    z[:, 0, 1] = 3.25 - (25 + 200 * torch.rand(B, generator=g, device="cuda")) * temperature
    x = torch.ones(B, 1, dtype=torch.int32, device="cuda")
    noise = torch.ones(B, V, device="cuda")
    r = ops.verify_drafts(z, x, torch.zeros(B, 1, device="cuda"), noise, temperature=temperature)
    assert (r.accepted == 1).all() and (r.tokens[:, 0] == 1).all() and (r.tokens[:, 1] == 0).all()
    s = z.double() / temperature
    lp = s - torch.logsumexp(s, 2, keepdim=True)
    want = torch.stack([lp[:, 0, 1], lp[:, 1, 0]], 1)
    # half a step of the result; the draft's own term is below e^-25 of the sum, and what else is lost below 2^-40
    tol = 2.0 ** -24 * want.abs() + math.exp(-25) + 2.0 ** -36
    assert ((r.logp.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("width", [256, 255, 40, 7])
@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("k", [3, 6])
def test_a_router_with_nan_shows_in_what_it_combines(k, dtype, width):
    # a token whose logits hold NaN or +inf has no expert, and NaN weights: its output is not 0
    T, E = 50, 16
    g = gen(k)
    z = torch.randn(T, E, generator=g, device="cuda")
    z[3, 2], z[20, 0] = math.nan, math.inf
    z[7] = -math.inf                                         # no expert is allowed: nothing is added
    r = ops.route(z, k)
    assert (r.experts[[3, 20, 7]] == -1).all() and r.weights[[3, 20]].isnan().all() and (r.weights[7] == 0).all()
    x = torch.randn(T, width, generator=g, device="cuda").to(dtype)
    y = ops.dispatch(x, r.place, r.offsets)
    for kind in {dtype, F}:
        for stream in (None, torch.cuda.current_stream()):
            out = ops.combine(y, r.place, r.weights, out_dtype=kind, stream=stream)
            assert out[[3, 20]].isnan().all() and (out[7] == 0).all()
            rest = torch.ones(T, dtype=torch.bool, device="cuda")
            rest[[3, 20]] = False
            assert out[rest].isfinite().all()
    # an entry that was dropped adds nothing where its weight is finite
    place = r.place.clone()
    place[5, 1] = -1
    w = r.weights[5].double()
    w[1] = 0
    got, each = ops.combine(y, place, r.weights, out_dtype=F)[5].double(), y[r.place[5].long()].double()
    # k products, each sum rounded, by half a step of the sum of their sizes
    assert ((got - (w[:, None] * each).sum(0)).abs() <= (k + 1) * 2.0 ** -24 * (w[:, None] * each).abs().sum(0)).all()


def test_kept_results_hold_no_workspace():
    z, x, u, noise, q, ok = make(200, 5, 1000, BF, F, True, 1.0, 1)
    for stream in (None, torch.cuda.current_stream()):
        held = lambda r: max(t.untyped_storage().nbytes() for t in r)  # noqa: E731
        own = lambda r: sum(-(-t.numel() * t.element_size() // 256) * 256 for t in r)  # noqa: E731
        r = ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok, stream=stream)
        assert held(r) <= own(r) + 8192
        logits = torch.randn(3000, 200, generator=gen(1), device="cuda")
        r = ops.route(logits, 2, stream=stream)
        assert held(r) <= own(r) + 8192
        r = ops.sort_by_group(r.experts, 200, stream=stream)
        assert held(r) <= own(r) + 8192
        r = ops.grad_norm([torch.ones(3000, device="cuda") for _ in range(500)], 1.0, stream=stream)
        assert held(r) <= own(r) + 8192


def test_noting_calls_leaves_calls_on_the_gpu_alone():
    from paper_1903_05133_gb300 import _lib
    host = _lib.host()
    z = torch.randn(6, 20, generator=gen(1), device="cuda")
    want = ops.route(z, 3)
    host.pretend(True)
    try:
        got = ops.route(z, 3)
        norm = ops.grad_norm([torch.full((4,), 3.0, device="cuda")]).norm
    finally:
        noted = host.pretend(False)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and norm.item() == 6.0 and noted is None
