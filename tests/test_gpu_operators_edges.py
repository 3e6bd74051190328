"""The operators at the edges of their domains, on the GPU: values, lengths and arguments where a formula
that holds elsewhere can fail."""
import math

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF, U, assert_within, close, gen, offsets_of, product_bound, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("T,V", [(1, 2), (5, 40), (3, 500), (4, 1500), (1300, 700), (3, 5000), (400, 2500), (1, 70001)])
def test_zeros_of_both_signs_are_equal_logits(T, V, dtype):
    # the alternatives go by index among them: every kernel that ranks, and the clusters of one row
    g = gen(T + V)
    z = torch.where(torch.rand(T, V, generator=g, device="cuda") < 0.5, -0.0, 0.0)
    z = torch.where(torch.rand(T, V, generator=g, device="cuda") < 0.2, -1.0, z).to(dtype)
    z[0, 0], z[0, 1] = -0.0, 0.0
    assert z[0, 0].signbit() and not z[0, 1].signbit()
    t = torch.zeros(T, dtype=torch.int32, device="cuda")
    for top in (1, 2, 32):
        r = ops.token_logprobs(z, t, top=top)
        order = torch.sort(z.double().abs(), dim=1, stable=True).indices[:, :top]     # 0 before 1, by index
        assert torch.equal(r.top_index[:, :order.shape[1]].long(), order)
    assert r.lse.isfinite().all() and r.entropy.isfinite().all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_gradients_whose_squares_overflow(bits):
    # v is infinite then and the step 0; the same at the last gradients whose squares are finite
    n = 1024
    g = torch.full((n,), 1e-3, device="cuda")
    g[256:512] = 1e21
    g[512:768] = -3e38
    g[768:] = 5e19                                          # v = 2.5e36
    p = torch.ones(n, device="cuda")
    copy = torch.zeros(n, dtype=BF, device="cuda")
    o = ops.AdamW([p], bits=bits, copies=[copy])
    o.step([g], lr=0.125)
    assert (p[256:768] == 1).all() and (copy == p.to(BF)).all()
    # elsewhere the first step is lr times the gradient's sign
    assert (p[:256] - 0.875).abs().max() < 1e-5 and (p[768:] - 0.875).abs().max() < 1e-5
    if bits == 32:
        assert (o.v[256:768] == math.inf).all() and o.m.isfinite().all() and o.v[768:].isfinite().all()
        o.step([torch.zeros(n, device="cuda")], lr=0.125)
        assert p.isfinite().all() and (p[256:768] == 1).all()
    bad = torch.ones(n, device="cuda")
    ops.AdamW([bad], bits=bits).step([torch.full((n,), math.inf, device="cuda")], lr=0.1)
    assert bad.isnan().all()                                # infinity over infinity


def test_adamw_second_moments_below_the_normal_numbers():
    # sqrt(v) of a denormal v; eps is small enough for it to count
    g = (torch.arange(1, 4097, device="cuda") * 1e-22).float()
    p = torch.zeros(4096, device="cuda")
    o = ops.AdamW([p], eps=1e-30, beta2=0.999)
    o.step([g], lr=1.0)
    v = o.v.double()
    # the products' and the sum's rounding steps are 2^-149 there
    assert ((v - 0.001 * g.double() ** 2).abs() <= 2.0 ** -147 + 2.0 ** -20 * v).all() and (v[:1000] < 1.17e-38).all()
    some = v > 0
    m = 0.1 * g.double()
    want = -(m / 0.1) / ((v / 0.001).sqrt() + 1e-30)
    off = (p.double() - want).abs()[some] / want.abs()[some]
    assert some.sum() > 2000 and off.max() <= 2.0 ** -19, off.max()
    assert p.isfinite().all()


def check_far_apart(z, t, top, temperature, allowed=None):
    # as check_logprobs, with a reference that takes the largest logit away before it divides: next to
    # a log-sum-exp of 1e20 even 64 bits do not see the others
    V = z.shape[1]
    r = ops.token_logprobs(z, t, top=top, temperature=temperature, allowed=allowed)
    raw = z.double()
    ok = raw > -1e30
    if allowed is not None:
        ok = ok & allowed
    raw = raw.masked_fill(~ok, -math.inf)
    m = raw.amax(1, keepdim=True)
    none = m.isinf()
    d = ((raw - m) / temperature).masked_fill(~ok, -math.inf)
    log_s = torch.logsumexp(d, 1, keepdim=True)
    lp = torch.where(ok, d - log_s, -math.inf)
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    lse = torch.where(none, -math.inf, m / temperature + log_s)[:, 0]
    logp = lp.gather(1, t.long()[:, None])[:, 0]
    s = 2.0 ** -24 * (V / 512 + 64)                         # check_logprobs's bounds
    size = lambda v: torch.where(v.isinf(), 0.0, v.abs())  # noqa: E731
    close(r.lse, lse, s + 2.0 ** -22 * size(lse))
    close(r.logp, logp, s + 2.0 ** -22 * (size(logp) + 1))
    close(r.entropy, ent, (2 * s + 2.0 ** -22) * (1 + ent))
    if top:
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :top]
        best = lp.gather(1, order)
        assert torch.equal(r.top_index[:, :order.shape[1]].long(), torch.where(best.isinf(), -1, order))
        close(r.top_logp[:, :order.shape[1]], best, s + 2.0 ** -22 * (size(best) + 1))
    return r


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("T,V", [(4, 3), (5, 300), (3, 1800), (1300, 1000), (3, 9000), (400, 3000), (1, 70001)])
def test_logprobs_tiny_temperatures(T, V, dtype):
    # the distances to the largest logit, in units of the temperature, pass fp32's range
    g = gen(T * 5 + V)
    z = torch.randint(-1, 2, (T, V), generator=g, device="cuda").to(dtype)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    ok = torch.rand(T, V, generator=g, device="cuda") < 0.5
    ok[0] = False
    for temperature in (1e-8, 1e-20, 2e-38):
        check_far_apart(z, t, 5, temperature)
        r = check_far_apart(z, t, 5, temperature, allowed=ok)
        assert r.entropy[0] == 0 and r.lse[0] == -math.inf
        check_far_apart(z.masked_fill(~ok, -math.inf), t, 0, temperature)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("T,V", [(4, 3), (5, 300), (1300, 1000), (3, 9000), (400, 3000), (1, 70001)])
def test_logprobs_logits_at_the_ends_of_fp32(T, V, dtype):
    z = torch.zeros(T, V, device="cuda")
    z[:, V // 2] = 3e38
    if T > 1:
        z[T - 1] = -3e29
    z = z.to(dtype)
    t = torch.full((T,), V // 2, device="cuda")
    r = check_far_apart(z, t, 3, 1.0)
    assert (r.entropy[:max(T - 1, 1)] == 0).all() and (r.logp[:max(T - 1, 1)] == 0).all()


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("T,V", [(3, 10), (1300, 600), (2, 5000)])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient_of_a_target_that_is_no_class(T, V, dtype, entropy):
    # as its log probability: NaN, and only in its row; a target below 0 has none
    g = gen(V)
    z = randn(g, T, V, dtype=dtype, std=2.0)
    ok = torch.rand(T, V, generator=g, device="cuda") < 0.7
    ok[:, 0] = True
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[0], t[1] = V, -3
    ones = torch.ones(T, device="cuda")
    for allowed in (None, ok):
        f = ops.token_logprobs(z, t, allowed=allowed)
        assert f.logp[0].isnan() and f.logp[1] == 0
        d = ops.token_logprobs_backward(z, t, f.lse, f.entropy, ones, ones if entropy else None, allowed=allowed)
        assert d[1:].isfinite().all()
        if allowed is None:
            assert d[0].isnan().all()
        else:
            assert d[0][ok[0]].isnan().all() and (d[~ok] == 0).all()


@pytest.mark.parametrize("T,K,N,off", [
    (100, 64, 40, [0, 50, 20]), (100, 72, 136, [0, 30, 10, 200]), (200, 96, 72, [-5, 30, 10, 1000]),
    (9, 2056, 130, [0, 5, 3, 4, 9, 2]), (700, 512, 520, [100, 400, 50, 350, 600, 20]), (3000, 264, 2568, [7, 2500, 1, 2999, 2000]),
    (640, 80, 24, [(i * 37) % 641 for i in range(70)]), (5000, 136, 264, [4000 - i if i % 3 else i for i in range(40)])])
@pytest.mark.parametrize("out", [BF, F])
def test_offsets_that_go_back_leave_each_row_to_its_first_group(T, K, N, off, out):
    g = gen(T + K)
    G = len(off) - 1
    at = torch.tensor(off, dtype=torch.int32, device="cuda")
    owner, top = [-1] * T, 0
    clamped = [min(max(o, 0), T) for o in off]
    for i in range(G):
        top = max(top, clamped[i])
        for r in range(top, clamped[i + 1]):
            owner[r] = i
    x, w = randn(g, T, K, dtype=BF), randn(g, G, N, K, dtype=BF, std=K ** -0.5)
    dy = randn(g, T, N, dtype=BF)
    h = randn(g, T, K, dtype=BF)
    first = None
    for _ in range(3):
        y = ops.grouped_product(x, w, at, out=torch.full((T, N), 9.0, dtype=out, device="cuda"))
        dx = ops.grouped_product_dx(dy, w, at, h=h, out=torch.full((T, K), 9.0, dtype=out, device="cuda"))
        assert first is None or (torch.equal(first[0], y) and torch.equal(first[1], dx))
        first = y, dx
    for i in range(-1, G):
        rows = torch.tensor([r for r in range(T) if owner[r] == i], device="cuda", dtype=torch.int64)
        if i < 0:
            assert (y[rows] == 0).all() and (dx[rows] == 0).all()
        elif len(rows):
            m = w[i].double()
            assert_within(y[rows], x[rows].double() @ m.T, product_bound(x[rows].double() @ m.T, x[rows].double().abs() @ m.T.abs(), K, out))
            ref = dy[rows].double() @ m
            assert_within(dx[rows], ref * (h[rows] > 0), product_bound(ref, dy[rows].double().abs() @ m.abs(), N, out))
    ops.operator_check()


@pytest.mark.parametrize("N,K,step", [(24, 64, 8), (24, 64, 64), (130, 72, 72), (1, 64, 8), (300, 128, 128), (40, 64, 0)])
def test_weights_whose_groups_overlap(N, K, step):
    # windows of one buffer, `step` further on for each group, and the groups' rows in turn
    g = gen(N + step)
    sizes = [3, 0, 70, 41]
    T, off = sum(sizes), offsets_of(sizes)
    flat = randn(g, 3 * step + N * K, dtype=BF)
    turn = randn(g, N, 4 * K, dtype=BF)
    x, dy = randn(g, T, K, dtype=BF), randn(g, T, N, dtype=BF)
    for w in (flat.as_strided((4, N, K), (step, K, 1)), turn.as_strided((4, N, K), (K, 4 * K, 1))):
        own = w.contiguous()
        assert torch.equal(ops.grouped_product(x, w, off), ops.grouped_product(x, own, off))
        assert torch.equal(ops.grouped_product_dx(dy, w, off), ops.grouped_product_dx(dy, own, off))
    ops.operator_check()


@pytest.mark.parametrize("dtype", [HF, BF])
def test_product_dw_long_sums_keep_their_precision(dtype):
    # 2^20 rows of one group among 40 that are too many tiles to be summed in parts.  Every product is
    # positive, so that an addition that truncates is off the same way every time.  The bound does not
    # grow with the length: the result's rounding, and those of sums of a few thousand products.
    g = gen(40)
    sizes = [3] * 40
    sizes[7] = 1 << 20
    T, N, K = sum(sizes), 40, 24
    dy = (torch.rand(T, N, generator=g, device="cuda") * 0.2 + 0.1).to(dtype)
    x = (torch.rand(T, K, generator=g, device="cuda") * 0.2 + 0.1).to(dtype)
    dw = ops.grouped_product_dw(dy, x, offsets_of(sizes))
    a, b = dy[21:21 + sizes[7]].double(), x[21:21 + sizes[7]].double()
    ref = a.T @ b
    assert ref.max() < 65000
    assert ((dw[7].double() - ref).abs() <= (U[dtype] + 2.0 ** -14) * ref).all(), ((dw[7].double() - ref).abs() / ref).max()
    ref = dy[:3].double().T @ x[:3].double()
    assert ((dw[0].double() - ref).abs() <= (U[dtype] + 2.0 ** -20) * ref).all()
    ops.operator_check()


@pytest.mark.parametrize("T,N", [(3, 136), (300, 136), (1024, 2560)])
@pytest.mark.parametrize("dx", [False, True])
def test_product_long_sums_keep_their_precision(T, N, dx):
    # the same of the rows' products: by clusters, by single CTAs and by pairs, K = 2^18
    g = gen(T)
    K = 1 << 18
    x = torch.rand(T, K, generator=g, device="cuda", dtype=HF) * 0.4 + 0.2
    w = torch.rand(2, N, K, generator=g, device="cuda", dtype=HF) * 0.4 + 0.2
    off = offsets_of([T // 3, T - T // 3])
    if dx:
        y = ops.grouped_product_dx(x, w.transpose(1, 2).contiguous(), off)
    else:
        y = ops.grouped_product(x, w, off)
    for g0, rows in ((0, slice(0, 1)), (1, slice(T - 2, T))):
        ref = x[rows].double() @ w[g0].double().T
        assert ((y[rows].double() - ref).abs() <= (2.0 ** -11 + 2.0 ** -14) * ref).all(), ((y[rows].double() - ref).abs() / ref).max()
    ops.operator_check()


@pytest.mark.parametrize("N,K", [(72, 40), (264, 520)])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (HF, F)])
def test_product_dw_every_end_of_a_group(N, K, dtype, out):
    # all lengths to two chunks and a row, each group between groups of values that may not reach it; the
    # same to the bit every time
    g = gen(N + K)
    sizes = [n for k in range(130) for n in (k, 1 + k % 17)]
    T = sum(sizes)
    dy, x = randn(g, T, N, dtype=dtype), randn(g, T, K, dtype=dtype)
    at = [0]
    for n in sizes:
        at.append(at[-1] + n)
    for i in range(1, len(sizes), 2):
        dy[at[i]:at[i + 1]], x[at[i]:at[i + 1]] = math.nan, math.inf
    off = offsets_of(sizes)
    dw, db = ops.grouped_product_dw(dy, x, off, bias_grad=True, out_dtype=out)
    for i in range(0, len(sizes), 2):
        a, b = dy[at[i]:at[i + 1]].double(), x[at[i]:at[i + 1]].double()
        assert_within(dw[i], a.T @ b, product_bound(a.T @ b, a.abs().T @ b.abs(), sizes[i], out))
        assert_within(db[i], a.sum(0), (sizes[i] + 16) * 2.0 ** -24 * a.abs().sum(0) + 1e-300)
    assert dw[1::2].isnan().all() and db[1::2].isnan().all()
    even = dw[0::2].clone()
    for _ in range(10):
        again = ops.grouped_product_dw(dy, x, off, out_dtype=out)
        assert torch.equal(again[0::2], even)
    ops.operator_check()


@pytest.mark.parametrize("sizes,K,N", [([3, 0, 2], 4096, 128), ([300, 1, 513], 512, 264), ([90, 40], 77, 51), ([20, 31], 264, 72)])
def test_product_dx_into_the_mask_itself(sizes, K, N):
    g = gen(K + N)
    T, G = sum(sizes), len(sizes)
    dy, w, h = randn(g, T, N, dtype=BF), randn(g, G, N, K, dtype=BF), randn(g, T, K + 8, dtype=BF)[:, 8:]
    off = offsets_of(sizes)
    want = ops.grouped_product_dx(dy, w, off, h=h)
    assert ops.grouped_product_dx(dy, w, off, h=h, out=h) is h and torch.equal(h, want)
