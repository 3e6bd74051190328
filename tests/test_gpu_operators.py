"""Grouped products, token log probabilities and AdamW on the GPU, each against its definition in
64 bits.  The bounds are those of the arithmetic: u is the unit roundoff of the result's type, and
a sum of n fp32 terms is off by at most n rounding steps of the sum of their magnitudes (the tensor
cores add 16 products at a time and truncate, so a step counts twice)."""
import math

import numpy as np
import pytest
import torch

from paper_1903_05133_gb300 import operators as ops

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


# ------------------------------------------------------------------ grouped products
def offsets_of(sizes):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")


def product_bound(ref, mag, length, dtype):
    steps = (min(length, 1024) if dtype == F else length) / 16 + length / 1024 + 8
    return U[dtype] * ref.abs() + 2 * steps * 2.0 ** -23 * mag + TINY[dtype] + 1e-300


def assert_within(got, ref, bound):
    off = (got.double() - ref).abs()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert got.shape == ref.shape and not got.isnan().any() and worst <= 1.0, worst


def ref_rows(a, w, sizes, transpose):
    """Rows of a times each group's matrix, and the same of the magnitudes, in 64 bits."""
    ys, ms, t = [], [], 0
    for g, n in enumerate(sizes):
        x, m = a[t:t + n].double(), w[g].double()
        m = m.T if transpose else m
        ys.append(x @ m)
        ms.append(x.abs() @ m.abs())
        t += n
    return torch.cat(ys), torch.cat(ms)


# sizes of the groups, inner, outer: single rows, empty groups, ends inside tiles, one group of
# several tiles, widths that are no multiple of 8, 64 or 128
ROWS = [([1], 64, 128), ([1, 0, 1, 0], 72, 40), ([0, 0, 5], 200, 136), ([17, 33, 64, 0, 1, 15], 264, 200),
        ([300, 1, 513], 512, 264), ([257], 1096, 130), ([64] * 5, 64, 10), ([3, 129, 70], 77, 51),
        ([255, 256, 257], 128, 384), ([2], 8, 1), ([40, 0, 9], 1, 9), ([700], 2056, 520)]


@pytest.mark.parametrize("sizes,K,N", ROWS)
@pytest.mark.parametrize("dtype,out", [(BF, BF), (HF, HF), (BF, F)])
def test_product(sizes, K, N, dtype, out):
    g = gen(K * 7 + N)
    T, G = sum(sizes), len(sizes)
    x, w = randn(g, T, K, dtype=dtype), randn(g, G, N, K, dtype=dtype, std=K ** -0.5)
    bias = randn(g, G, N)
    off = offsets_of(sizes)
    ref, mag = ref_rows(x, w, sizes, True)
    assert_within(ops.grouped_product(x, w, off, out_dtype=out), ref, product_bound(ref, mag, K, out))
    b = torch.cat([bias[i].double().expand(n, N) for i, n in enumerate(sizes)])
    y = ops.grouped_product(x, w, off, bias=bias, relu=True, out_dtype=out)
    pre = ref + b
    assert_within(y, pre.clamp(min=0), product_bound(pre, mag + b.abs(), K + 16, out))
    ops.operator_check()


@pytest.mark.parametrize("sizes,K,N", ROWS)
@pytest.mark.parametrize("dtype,out", [(BF, BF), (HF, HF), (HF, F)])
def test_product_dx(sizes, K, N, dtype, out):
    g = gen(K * 11 + N)
    T, G = sum(sizes), len(sizes)
    dy, w = randn(g, T, N, dtype=dtype), randn(g, G, N, K, dtype=dtype, std=N ** -0.5)
    h = randn(g, T, K, dtype=dtype).clamp(min=0)
    off = offsets_of(sizes)
    ref, mag = ref_rows(dy, w, sizes, False)
    assert_within(ops.grouped_product_dx(dy, w, off, out_dtype=out), ref, product_bound(ref, mag, N, out))
    got = ops.grouped_product_dx(dy, w, off, h=h, out_dtype=out)
    assert_within(got, ref * (h > 0), product_bound(ref, mag, N, out))
    assert (got[h <= 0] == 0).all()
    ops.operator_check()


@pytest.mark.parametrize("sizes,K,N", ROWS + [([0], 24, 16), ([0, 0], 130, 7), ([5000], 64, 64)])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (HF, HF), (BF, F)])
def test_product_dw(sizes, K, N, dtype, out):
    g = gen(K * 13 + N)
    T = sum(sizes)
    dy, x = randn(g, T, N, dtype=dtype), randn(g, T, K, dtype=dtype)
    dw, db = ops.grouped_product_dw(dy, x, offsets_of(sizes), bias_grad=True, out_dtype=out)
    t = 0
    for i, n in enumerate(sizes):
        a, b = dy[t:t + n].double(), x[t:t + n].double()
        ref, mag = a.T @ b, a.abs().T @ b.abs()
        assert_within(dw[i], ref, product_bound(ref, mag, n, out))
        assert_within(db[i], a.sum(0), (n + 16) * 2.0 ** -24 * a.abs().sum(0) + 1e-300)
        t += n
    assert torch.equal(dw, ops.grouped_product_dw(dy, x, offsets_of(sizes), out_dtype=out))
    ops.operator_check()


@pytest.mark.parametrize("G,N,K", [(40, 1300, 1101), (30, 7, 205), (9, 130, 9)])
def test_product_unaligned_weights_of_empty_groups(G, N, K):
    g = gen(G + N + K)
    sizes = [0] * G
    sizes[3], sizes[4], sizes[G - 1] = 2, 1, 5
    T = sum(sizes)
    x, w = randn(g, T, K, dtype=BF), randn(g, G, N, K, dtype=BF, std=K ** -0.5)
    dy = randn(g, T, N, dtype=BF)
    off = offsets_of(sizes)
    w[0] = w[5] = math.nan                                  # in groups without rows
    used = [3, 4, G - 1]
    ref, mag = ref_rows(x, w[used], [2, 1, 5], True)
    assert_within(ops.grouped_product(x, w, off), ref, product_bound(ref, mag, K, BF))
    ref, mag = ref_rows(dy, w[used], [2, 1, 5], False)
    assert_within(ops.grouped_product_dx(dy, w, off, out_dtype=F), ref, product_bound(ref, mag, N, F))
    off = off.clone()                                       # outside the rows on both sides
    off[0], off[G] = -4, T + 100
    ref, mag = ref_rows(x, w[used], [2, 1, 5], True)
    assert_within(ops.grouped_product(x, w, off)[2:], ref[2:], product_bound(ref, mag, K, BF)[2:])
    ops.operator_check()


# few tiles and long sums: the CTAs of a cluster share a tile, over more tiles than clusters, columns
# that do not divide among them, groups of several tiles, and CTAs without a column
@pytest.mark.parametrize("sizes,K,N", [([5], 4104, 2432), ([1], 8192, 64), ([63, 1], 8200, 300), ([0, 31], 2056, 136),
                                       ([200], 4096, 520), ([150, 3, 90], 4400, 56), ([2, 3, 1, 0, 9], 2048, 480)])
@pytest.mark.parametrize("out", [BF, F])
def test_product_shared_tiles(sizes, K, N, out):
    g = gen(K * 19 + N)
    T, G = sum(sizes), len(sizes)
    x, w = randn(g, T, K, dtype=BF), randn(g, G, N, K, dtype=BF, std=K ** -0.5)
    off = offsets_of(sizes)
    ref, mag = ref_rows(x, w, sizes, True)
    y = ops.grouped_product(x, w, off, out_dtype=out)
    assert_within(y, ref, product_bound(ref, mag, K, out))
    wt = w.transpose(1, 2).contiguous()                     # the same sums as a gradient
    h = randn(g, T, N, dtype=BF)
    got = ops.grouped_product_dx(x, wt, off, h=h, out_dtype=out)
    assert_within(got, ref * (h > 0), product_bound(ref, mag, K, out))
    for _ in range(3):
        assert torch.equal(y, ops.grouped_product(x, w, off, out_dtype=out))
    ops.operator_check()


@pytest.mark.parametrize("sizes,K,N", [([3000, 0, 1500, 70, 2001], 72, 130), ([8192], 520, 264), ([1, 9000, 0], 77, 3),
                                       ([2049], 1, 1), ([1100] * 7, 300, 40)])
@pytest.mark.parametrize("dtype,out", [(BF, BF), (HF, F)])
def test_product_dw_long_groups(sizes, K, N, dtype, out):
    # few tiles over many rows: summed in parts
    g = gen(K * 17 + N)
    T, G = sum(sizes), len(sizes)
    dy, x = randn(g, T, N, dtype=dtype), randn(g, T, K, dtype=dtype)
    into = torch.full((G, N, K + 3), 7.0, dtype=out, device="cuda")
    dw, db = ops.grouped_product_dw(dy, x, offsets_of(sizes), bias_grad=True, out=into[:, :, :K])
    t = 0
    for i, n in enumerate(sizes):
        a, b = dy[t:t + n].double(), x[t:t + n].double()
        assert_within(dw[i], a.T @ b, product_bound(a.T @ b, a.abs().T @ b.abs(), n, out))
        assert_within(db[i], a.sum(0), (n + 16) * 2.0 ** -24 * a.abs().sum(0) + 1e-300)
        t += n
    assert (into[:, :, K:] == 7).all()
    assert torch.equal(dw, ops.grouped_product_dw(dy, x, offsets_of(sizes), out_dtype=out))
    # offsets outside the rows, and one that goes back: its group is empty
    off = torch.tensor([-5, T // 2, T // 4, T + 9], dtype=torch.int32, device="cuda")
    dw = ops.grouped_product_dw(dy, x, off, out_dtype=F)
    for i, (b, e) in enumerate(((0, T // 2), (0, 0), (T // 4, T))):
        a, b = dy[b:e].double(), x[b:e].double()
        assert_within(dw[i], a.T @ b, product_bound(a.T @ b, a.abs().T @ b.abs(), T, F))
    ops.operator_check()


def test_product_many_groups_and_folds():
    # more groups than a warp's scan takes at once, and sums of several folded segments
    g = gen(3)
    sizes = [(i * 37) % 11 for i in range(300)]
    T, K, N = sum(sizes), 2500, 72
    x, w = randn(g, T, K, dtype=BF), randn(g, len(sizes), N, K, dtype=BF, std=0.02)
    ref, mag = ref_rows(x, w, sizes, True)
    assert_within(ops.grouped_product(x, w, offsets_of(sizes), out_dtype=F), ref, product_bound(ref, mag, K, F))


@pytest.mark.parametrize("K,N", [(128, 256), (77, 51)])
def test_product_strides(K, N):
    # rows, weights and results inside larger buffers, at odd places; one matrix for all groups
    g = gen(5)
    sizes = [30, 0, 71]
    T, off = 101, offsets_of([30, 0, 71])
    for pad, shift in ((8, 8), (3, 1)):
        X = randn(g, T, K + pad + shift, dtype=BF)[:, shift:shift + K]
        W = randn(g, 3, N + 2, K + pad + shift, dtype=BF, std=0.1)[:, 1:N + 1, shift:shift + K]
        big = torch.full((T + 2, N + pad + shift), float("nan"), dtype=BF, device="cuda")
        y = big[1:T + 1, shift:shift + N]
        assert ops.grouped_product(X, W, off, out=y) is y
        ref, mag = ref_rows(X, W, sizes, True)
        assert_within(y, ref, product_bound(ref, mag, K, BF))
        dX = ops.grouped_product_dx(y, W, off)
        rdx, mdx = ref_rows(y, W, sizes, False)
        assert_within(dX, rdx, product_bound(rdx, mdx, N, BF))
        out = torch.full((3, N, K + pad), float("nan"), dtype=F, device="cuda")
        ops.grouped_product_dw(y, X, off, out=out[:, :, :K])
        rdw = y[30:].double().T @ X[30:].double()
        assert_within(out[2, :, :K], rdw, product_bound(rdw, y[30:].double().abs().T @ X[30:].double().abs(), 71, F))
        assert (out[1, :, :K] == 0).all() and out[:, :, K:].isnan().all()
        big[1:T + 1, shift:shift + N] = float("nan")
        assert big.isnan().all()                          # nothing outside the window changed
    # aligned rows whose width is not: what lies between them is not read
    wide = -(-max(K, N) // 8) * 8 + 8
    X = torch.full((T, wide), float("nan"), dtype=BF, device="cuda")[:, :K].copy_(randn(g, T, K, dtype=BF))
    W = torch.full((3, N, wide), float("nan"), dtype=BF, device="cuda")[:, :, :K].copy_(randn(g, 3, N, K, dtype=BF))
    D = torch.full((T, wide), float("nan"), dtype=BF, device="cuda")[:, :N].copy_(randn(g, T, N, dtype=BF))
    for got, ref, n in ((ops.grouped_product(X, W, off), ref_rows(X, W, sizes, True), K),
                        (ops.grouped_product_dx(D, W, off), ref_rows(D, W, sizes, False), N),
                        (ops.grouped_product_dw(D, X, off)[2], (D[30:].double().T @ X[30:].double(), D[30:].double().abs().T @ X[30:].double().abs()), 71)):
        assert_within(got, ref[0], product_bound(ref[0], ref[1], n, BF))
    one = randn(g, N, K, dtype=BF)
    x = randn(g, T, K, dtype=BF)
    shared = ops.grouped_product(x, one.expand(3, N, K), off)
    assert torch.equal(shared, ops.grouped_product(x, one.expand(3, N, K).contiguous(), off))


def test_product_rows_of_no_group_and_bad_values_stay_apart():
    g = gen(9)
    T, K, N = 200, 96, 72
    x, w, dy = randn(g, T, K, dtype=BF), randn(g, 3, N, K, dtype=BF), randn(g, T, N, dtype=BF)
    x[20:50], dy[20:50] = float("nan"), float("inf")       # group 1's rows only
    w[1] = float("nan")
    off = torch.tensor([7, 20, 50, 180], dtype=torch.int32, device="cuda")
    for y in (ops.grouped_product(x, w, off, out=torch.full((T, N), 9.0, dtype=BF, device="cuda")),
              ops.grouped_product_dx(dy, w, off, out=torch.full((T, K), 9.0, dtype=BF, device="cuda"))):
        assert (y[:7] == 0).all() and (y[180:] == 0).all()
        assert y[7:20].isfinite().all() and y[50:180].isfinite().all() and y[20:50].isnan().all()
    dw, db = ops.grouped_product_dw(dy, x, off, bias_grad=True)
    assert dw[0].isfinite().all() and dw[2].isfinite().all() and dw[1].isnan().all()
    assert db[0].isfinite().all() and db[2].isfinite().all() and (db[1] == float("inf")).all()
    # offsets outside the rows, or going back: clamped, and an empty group
    odd = torch.tensor([-5, 30, 10, 1000], dtype=torch.int32, device="cuda")
    x = randn(g, T, K, dtype=BF)
    w = randn(g, 3, N, K, dtype=BF)
    y = ops.grouped_product(x, w, odd)
    ref, mag = ref_rows(x[10:], w[2:], [190], True)
    assert_within(y[30:], ref[20:], product_bound(ref, mag, K, BF)[20:])
    ops.operator_check()


def test_product_gradients_are_differences():
    # loss = sum(r * relu(x W^T + b)) in 64 bits, perturbed entry by entry
    g = gen(21)
    sizes, K, N = [5, 0, 9], 24, 16
    x, w, r = randn(g, 14, K, dtype=BF), randn(g, 3, N, K, dtype=BF), randn(g, 14, N, dtype=BF)
    h = randn(g, 14, K, dtype=BF).clamp(min=0)
    off = offsets_of(sizes)
    loss = lambda a, m: (ref_rows(a, m, sizes, True)[0] * r.double()).sum().item()  # noqa: E731
    dx = ops.grouped_product_dx(r, w, off, out_dtype=F)
    dw = ops.grouped_product_dw(r, x, off, out_dtype=F)
    for t, k in ((0, 0), (4, 23), (5, 7), (13, 11)):
        a = x.double()
        b = a.clone()
        a[t, k] -= 0.5
        b[t, k] += 0.5
        assert abs((loss(b, w) - loss(a, w)) - dx[t, k].item()) <= 1e-4 * (1 + abs(dx[t, k].item()))
    for i, n, k in ((0, 0, 0), (1, 3, 3), (2, 15, 23), (2, 7, 1)):
        a = w.double()
        b = a.clone()
        a[i, n, k] -= 0.5
        b[i, n, k] += 0.5
        assert abs((loss(x, b) - loss(x, a)) - dw[i, n, k].item()) <= 1e-4 * (1 + abs(dw[i, n, k].item()))
    assert torch.equal(ops.grouped_product_dx(r, w, off, h=h, out_dtype=F), torch.where(h > 0, dx, 0.0))


def test_product_on_another_stream():
    g = gen(8)
    sizes = [100, 200]
    x, w, off = randn(g, 300, 512, dtype=BF), randn(g, 2, 384, 512, dtype=BF), offsets_of([100, 200])
    want = ops.grouped_product(x, w, off)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [ops.grouped_product(x, w, off, stream=side) for _ in range(5)]
    odd = ops.grouped_product(x[:, :509], w[:, :, :509], off, stream=side)      # through the workspace
    side.synchronize()
    assert all(torch.equal(y, want) for y in got)
    ref, mag = ref_rows(x[:, :509], w[:, :, :509], sizes, True)
    assert_within(odd, ref, product_bound(ref, mag, 509, BF))


# ------------------------------------------------------------------ log probabilities
def ref_logprobs(logits, targets, allowed, temperature):
    raw = logits.double()
    ok = raw > -1e30
    if allowed is not None:
        ok = ok & allowed
    z = (raw / temperature).masked_fill(~ok, -math.inf)
    lse = torch.logsumexp(z, 1)
    lp = torch.where(ok, z - lse[:, None], -math.inf)
    p = torch.where(ok, lp.exp(), 0.0)
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    t = targets.long()
    logp = torch.where(t < 0, 0.0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0])
    return logp, ent, lse, lp, p, ok


def close(got, ref, tol):
    got = got.double()
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf])
    assert ((got - ref).abs()[~inf] <= tol.expand_as(ref)[~inf]).all(), ((got - ref).abs()[~inf] / tol.expand_as(ref)[~inf]).max()


def check_logprobs(z, t, top, temperature=1.0, allowed=None, exact_ties=True):
    V = z.shape[1]
    r = ops.token_logprobs(z, t, top=top, temperature=temperature, allowed=allowed)
    logp, ent, lse, lp, p, ok = ref_logprobs(z, t, allowed, temperature)
    size = torch.where(lse.isinf(), 0.0, lse.abs())
    # the sum's relative error: V / 512 terms a thread, joins, and the exponentials' own (2 ulp)
    s = 2.0 ** -24 * (V / 512 + 64)
    close(r.lse, lse, s + 2.0 ** -22 * size)
    given = torch.where(logp.isinf(), 0.0, logp.abs())
    close(r.logp, logp, s + 2.0 ** -22 * (given + 1))
    close(r.entropy, ent, (2 * s + 2.0 ** -22) * (1 + ent))
    if not top:
        assert r.top_logp is None and r.top_index is None
        return r
    raw = z.double().masked_fill(~ok, -math.inf)
    order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :top]
    n = order.shape[1]
    best = lp.gather(1, order)
    want = torch.where(best.isinf(), -1, order)
    assert torch.equal(r.top_index[:, :n].long(), want)
    close(r.top_logp[:, :n], best, s + 2.0 ** -22 * (torch.where(best.isinf(), 0.0, best.abs()) + 1))
    assert (r.top_index[:, n:] == -1).all() and (r.top_logp[:, n:] == -math.inf).all()
    return r


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("T,V,top", [(1, 1, 1), (3, 2, 5), (5, 10, 3), (2, 1000, 32), (7, 4097, 1), (1, 128001, 20),
                                     (400, 333, 8), (3, 65536, 32), (2, 50021, 0), (1, 31, 32)])
def test_logprobs(T, V, top, dtype):
    g = gen(T * 31 + V)
    z = randn(g, T, V, dtype=dtype, std=3.0)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[T // 2] = -1
    check_logprobs(z, t, top)
    check_logprobs(z, t.int(), top, temperature=0.37)


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("V", [9, 640, 20000])
def test_logprobs_masks(V, dtype):
    g = gen(V)
    T = 12
    z = randn(g, T, V, dtype=dtype, std=3.0)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    ok = torch.rand(T, V, generator=g, device="cuda") < 0.3
    ok[3] = False                                  # an empty row
    ok[5] = False
    ok[5, V - 1] = True                            # one class
    t[6] = V - 1
    ok[6, V - 1] = False                           # a target that is not allowed
    z2 = z.clone()
    z2[~ok] = float("nan")                         # what is masked is not looked at
    r = check_logprobs(z2.where(ok, torch.zeros_like(z)), t, 4, allowed=ok)
    assert torch.equal(ops.token_logprobs(z2, t, top=4, allowed=ok).lse, r.lse)
    assert r.lse[3] == -math.inf and r.entropy[3] == 0 and (r.top_index[3] == -1).all()
    check_logprobs(z, t, 4, allowed=ok[0])         # one mask for all rows
    low = z.masked_fill(~ok, -math.inf)
    check_logprobs(low, t, 4)
    big = torch.zeros(T, V + 3, dtype=torch.bool, device="cuda")
    big[:, 1:V + 1] = ok                           # rows of the mask at odd places
    check_logprobs(z, t, 4, allowed=big[:, 1:V + 1])
    if dtype != HF:
        low = z.masked_fill(~ok, torch.finfo(dtype).min)
        r2 = check_logprobs(low, t, 4)
        assert r2.lse[3] == -math.inf


def test_logprobs_extremes():
    z = torch.zeros(6, 3000, device="cuda")
    z[0] = 80.0                                    # ties all the way
    z[1] = torch.arange(3000, device="cuda") / 10  # rising: every entry beats those before it
    z[2] = -torch.arange(3000, device="cuda") / 10
    z[3, 7] = 1e4                                  # one class takes all
    z[4] = -1e4
    z[5] = torch.arange(3000, device="cuda") % 3
    t = torch.tensor([0, 2999, 0, 8, 1, 2], device="cuda")
    check_logprobs(z, t, 32)
    check_logprobs(z.to(BF), t, 32)
    up = torch.arange(120000, device="cuda").float()[None] / 1e4
    check_logprobs(up, torch.tensor([5], device="cuda"), 32)
    check_logprobs(torch.ones(300, 20000, dtype=BF, device="cuda"), torch.zeros(300, dtype=torch.int32, device="cuda"), 32)
    for bad in (float("nan"), float("inf")):
        y = z.clone()
        y[2, 1234] = bad
        r = ops.token_logprobs(y, t, top=3)
        assert r.lse[2].isnan() and r.logp[2].isnan() and r.entropy[2].isnan()
        assert (r.top_index[2] == -1).all() and r.lse[[0, 1, 3, 4, 5]].isfinite().all()
    t[1] = 3000
    assert ops.token_logprobs(z, t).logp[1].isnan()
    none = ops.token_logprobs(z[:0], t[:0], top=2)
    assert none.logp.shape == (0,) and none.top_index.shape == (0, 2)


def check_grad(z, t, temperature=1.0, allowed=None, entropy=True, out=None):
    T = z.shape[0]
    g = gen(T)
    dlogp = randn(g, T)
    dent = randn(g, T) if entropy else None
    f = ops.token_logprobs(z, t, temperature=temperature, allowed=allowed)
    d = ops.token_logprobs_backward(z, t, f.lse, f.entropy, dlogp, dent, temperature=temperature,
                                    allowed=allowed, out=out)
    logp, ent, lse, lp, p, ok = ref_logprobs(z, t, allowed, temperature)
    lp = torch.where(ok, lp, 0.0)
    one = torch.zeros_like(p)
    one[torch.arange(T, device="cuda"), t.long().clamp(min=0)] = 1
    a = torch.where(t < 0, 0.0, dlogp.double())[:, None]
    b = dent.double()[:, None] if entropy else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
    ref = torch.where(ok, (one - p) * a - b * torch.where(p > 0, p * (lp + ent[:, None]), 0.0), 0.0) / temperature
    V = z.shape[1]
    size = torch.where(lse.isinf(), 0.0, lse.abs())[:, None]
    rel = 2.0 ** -24 * (V / 512 + 64) + 2.0 ** -21 * (1 + size + lp.abs())
    mag = p * (a.abs() + b.abs() * (lp.abs() + ent[:, None] + 1)) / temperature
    bound = U[z.dtype] * ref.abs() + rel * mag + 2.0 ** -22 * (one * a).abs() / temperature + TINY[z.dtype] + 1e-37
    assert_within(d, ref, bound)
    assert (d[~ok] == 0).all()
    return d, ref


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 10), (4, 1001), (2, 70001), (130, 77)])
def test_logprobs_gradient(T, V, dtype):
    g = gen(T + V)
    z = randn(g, T, V, dtype=dtype, std=3.0)
    t = torch.randint(-1, V, (T,), generator=g, device="cuda").int()
    check_grad(z, t)
    check_grad(z, t, temperature=1.7, entropy=False)
    ok = torch.rand(T, V, generator=g, device="cuda") < 0.5
    ok[T - 1] = False
    check_grad(z, t, allowed=ok, temperature=0.8)
    wide = torch.zeros(T, V + 5, dtype=dtype, device="cuda")
    check_grad(z, t, out=wide[:, 3:V + 3])
    assert (wide[:, :3] == 0).all() and (wide[:, V + 3:] == 0).all()
    y = z.clone()
    f = ops.token_logprobs(z, t)
    d = torch.ones(T, device="cuda")
    want = ops.token_logprobs_backward(z, t, f.lse, f.entropy, d)
    assert ops.token_logprobs_backward(y, t, f.lse, None, d, out=y) is y and torch.equal(y, want)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("T", [3, 1300])
@pytest.mark.parametrize("V", [1, 33, 64, 65, 300, 512, 513, 1000, 1025, 2048, 2049, 3000])
def test_logprobs_few_classes(T, V, dtype):
    # on both sides of each length at which a row is taken by another kernel, few rows and many
    g = gen(T + V)
    big = randn(g, T, V + 3, dtype=dtype, std=3.0)
    z = big[:, 1:V + 1]                                     # rows of unit stride at any alignment
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[1] = -1
    check_logprobs(z, t, 0, temperature=1.7)
    allowed = torch.rand(T, V, generator=g, device="cuda") < 0.4
    allowed[0] = False
    allowed[2, 1:] = False
    for top, ok in ((1, None), (20, None), (32, allowed), (4, allowed[1])):
        check_logprobs(z, t, top, allowed=ok)
    same = torch.ones(T, V, dtype=dtype, device="cuda")     # equal logits: by index
    check_logprobs(same, t, 5)
    z = z.clone()
    z[0, V // 2] = math.nan
    r = ops.token_logprobs(z, t, top=2)
    assert r.lse[0].isnan() and r.entropy[0].isnan() and (r.top_index[0] == -1).all() and not r.lse[1:].isnan().any()


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("T,V", [(1300, 10), (1300, 500), (1300, 1024), (1300, 1025), (3, 512), (3, 513), (2600, 33)])
def test_logprobs_gradient_few_classes(T, V, dtype):
    g = gen(T * 3 + V)
    z = randn(g, T, V + 1, dtype=dtype, std=3.0)[:, 1:]
    t = torch.randint(-1, V, (T,), generator=g, device="cuda")
    check_grad(z, t, temperature=0.9)
    ok = torch.rand(T, V, generator=g, device="cuda") < 0.5
    ok[0] = False
    wide = torch.zeros(T, V + 5, dtype=dtype, device="cuda")
    check_grad(z, t, allowed=ok, out=wide[:, 3:V + 3])
    check_grad(z, t, allowed=ok[1], entropy=False)
    assert (wide[:, :3] == 0).all() and (wide[:, V + 3:] == 0).all()


def test_logprobs_gradient_is_differences():
    g = gen(77)
    z = randn(g, 2, 40, std=2.0)
    t = torch.tensor([3, 17], device="cuda")
    d, _ = check_grad(z, t, temperature=1.3)
    gg = gen(2)
    a, b = randn(gg, 2).double(), randn(gg, 2).double()    # as check_grad draws them

    def loss(y):
        r = ref_logprobs(y, t, None, 1.3)
        return (a * r[0] + b * r[1]).sum().item()
    for i, j in ((0, 3), (0, 0), (1, 17), (1, 39)):
        lo, hi = z.double(), z.double()
        lo[i, j] -= 1e-4
        hi[i, j] += 1e-4
        assert abs((loss(hi) - loss(lo)) / 2e-4 - d[i, j].item()) < 1e-5


# ------------------------------------------------------------------ AdamW
def grid8():
    low = [k * 2.0 ** -9 for k in range(8)]
    return np.array(low + [(8 + k) / 8 * 2.0 ** e for e in range(-6, 9) for k in range(8)][:-1])


def ref_adamw(p, g, m, v, t, lr, decay, b1=0.9, b2=0.999, eps=1e-8):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    step = lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
    return p - lr * decay * p - step, m, v, step


SIZES = [[1], [255, 256, 257], [5000, 3, 4096], [4097, 1, 1, 100000], [7] * 100]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("grad", [F, BF, HF])
def test_adamw_32(sizes, grad):
    g = gen(len(sizes))
    ps = [randn(g, n) for n in sizes]
    cs = [torch.empty(n, dtype=BF, device="cuda") for n in sizes]
    decay = [0.1 * (i % 2) for i in range(len(sizes))]
    o = ops.AdamW(ps, decay=decay, copies=cs)
    scale = torch.tensor([0.5], device="cuda")
    ref = [(p.double(), torch.zeros_like(p).double(), torch.zeros_like(p).double()) for p in ps]
    for t in range(1, 4):
        gs = [randn(g, n, dtype=grad, std=0.1) for n in sizes]
        o.step(gs, lr=0.01, grad_scale=scale)
        at = 0
        for i, n in enumerate(sizes):
            p, m, v = ref[i]
            p, m, v, step = ref_adamw(p, gs[i].double() * 0.5, m, v, t, 0.01, decay[i])
            ref[i] = (p, m, v)
            u = 2.0 ** -24
            assert ((o.m[at:at + n].double() - m).abs() <= 4 * t * u * (m.abs() + 0.1)).all()
            assert ((o.v[at:at + n].double() - v).abs() <= 8 * t * u * v + 1e-40).all()
            # m cancels where the gradients' signs differ, so the step is off by its rounding over sqrt(v)
            off = 4 * t * u * (0.01 * 0.2 / (v.sqrt() + 1e-8) + step.abs() * 16 + p.abs() + 0.01)
            assert ((ps[i].double() - p).abs() <= off * 4).all()
            assert torch.equal(cs[i], ps[i].to(BF))
            at += -(-n // 256) * 256
    assert o.t == 3


def decode(codes, scale):
    return codes.float().double().view(-1, 256) * scale.double()[:, None]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("grad", [F, BF])
def test_adamw_8(sizes, grad):
    g = gen(len(sizes) + 50)
    ps = [randn(g, n) for n in sizes]
    cs = [torch.empty(n, dtype=HF, device="cuda") for n in sizes]
    o = ops.AdamW(ps, bits=8, decay=0.1, copies=cs)
    grid = torch.tensor(grid8(), device="cuda")
    blocks = [-(-n // 256) for n in sizes]

    def padded(ts):
        return torch.cat([torch.nn.functional.pad(t.double(), (0, b * 256 - t.numel())) for t, b in zip(ts, blocks)]).view(-1, 256)
    for t in range(1, 4):
        gs = [randn(g, n, dtype=grad, std=0.1) for n in sizes]
        before = padded(ps)
        m0, r0 = decode(o.m, o.m_scale), decode(o.root, o.root_scale)
        o.step(gs, lr=0.01, seed=t * 12345)
        p, m, v, step = ref_adamw(before, padded(gs), m0, r0 ** 2, t, 0.01, 0.1)
        after = padded(ps)
        assert ((after - p).abs() <= 2.0 ** -20 * (step.abs() + 0.01 * 0.2 * 2.0 ** -4 / (v.sqrt() + 1e-8)) + 2.0 ** -22 * p.abs()).all()
        for a, b in zip(cs, ps):
            assert torch.equal(a, b.to(HF))
        for code, scale, x, near in ((o.m, o.m_scale, m, True), (o.root, o.root_scale, v.sqrt(), False)):
            most = x.abs().amax(1)
            # the first moment's two terms may cancel: its rounding is theirs
            terms = (0.9 * m0).abs() + (0.1 * padded(gs)).abs() if near else x
            assert ((scale.double() - most / 448).abs() <= 2.0 ** -21 * terms.amax(1) / 448 + 1e-30 / 448).all()
            got = code.float().double().view(-1, 256)
            y = torch.where(scale[:, None] > 0, x / scale.double()[:, None], 0.0)
            k = (torch.searchsorted(grid, y.abs().clamp(max=448.0).contiguous(), right=True) - 1)
            lo, hi = grid[k], grid[(k + 1).clamp(max=len(grid) - 1)]
            # nearest: within half a step; at random: one of the two neighbours (with fp32's slack)
            slack = 2.0 ** -18 * torch.where(scale[:, None] > 0, terms / scale.double()[:, None], 0.0) + 1e-9
            err = (got - y).abs()
            assert (err <= torch.maximum((hi - lo) / (2 if near else 1), slack) + slack).all()
            if not near:
                assert ((got > 0) | (y <= 0)).all()
                assert (got[(y == 0)] == 0).all()


def codes_of(a, seed=None):
    """The 8-bit form of blocks of 256 fp32 values in elementary operations, each rounded to fp32."""
    most = a.abs().amax(1, keepdim=True)
    most = torch.where(most < 1e-30, 0.0, most)
    x = torch.where(most > 0, a * (most.reciprocal() * 448.0), 0.0)
    if seed is not None:
        j = (torch.arange(a.numel(), device="cuda") + (seed & 0xFFFFFFFF) * 0xBB67AE85) & 0xFFFFFFFF
        j = (j * 0x9E3779B9) & 0xFFFFFFFF
        j = ((j ^ (j >> 15)) * 0x6A09E667) & 0xFFFFFFFF
        r = ((j ^ (j >> 13)) >> 12).int().view(a.shape)
        low = torch.where(x < 2.0 ** -6, 2.0 ** -6, 0.0)
        t = (((x + low).view(torch.int32) + r) & ~0xFFFFF).view(torch.float32) - low
        x = torch.where(x > 0, t.clamp(min=2.0 ** -9), 0.0)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), most[:, 0] * (1.0 / 448.0)


def test_adamw_8_to_the_bit():
    # every code and scale equals that of the formula evaluated operation by operation in fp32: no
    # operations are contracted, and the square root is the rounded one
    g = gen(91)
    n = 256 * 20000
    p = randn(g, n)
    o = ops.AdamW([p], bits=8)
    scale = torch.tensor([0.7], device="cuda")
    for t in range(1, 4):
        gr = randn(g, n, dtype=BF, std=1e-3)
        m = o.m.float().view(-1, 256) * o.m_scale[:, None]
        r = o.root.float().view(-1, 256) * o.root_scale[:, None]
        v = r * r
        x = gr.float().view(-1, 256) * scale
        m = 0.9 * m + (1 - 0.9) * x
        v = 0.999 * v + (1 - 0.999) * x * x
        o.step([gr], lr=1e-3, grad_scale=scale, seed=t * 77)
        for (code, s), got, got_s in ((codes_of(m), o.m, o.m_scale), (codes_of(v.sqrt(), t * 77), o.root, o.root_scale)):
            assert torch.equal(got.view(torch.uint8), code.view(-1).view(torch.uint8))
            assert torch.equal(got_s, s)


def test_adamw_8_random_rounding_keeps_the_mean_and_repeats():
    n = 256 * 400
    p = torch.zeros(n, device="cuda")
    g = torch.full((n,), 0.5, device="cuda")
    g[::256] = 1.0                                        # the block's largest
    o = ops.AdamW([p], bits=8, beta2=0.9)
    o.step([g], lr=0.0, seed=1)
    want = math.sqrt(0.1) * 0.5
    r = decode(o.root, o.root_scale).view(-1)[1:256]      # 0.5 of the largest is on the grid
    assert ((r - want).abs() < 1e-6).all()
    g = torch.full((n,), 0.53, device="cuda")
    g[::256] = 1.0
    a, b = ops.AdamW([p], bits=8, beta2=0.9), ops.AdamW([p], bits=8, beta2=0.9)
    a.step([g], lr=0.0, seed=7)
    b.step([g], lr=0.0, seed=7)
    assert torch.equal(a.root.view(torch.uint8), b.root.view(torch.uint8))
    root = decode(a.root, a.root_scale)[:, 1:].reshape(-1)
    want = math.sqrt(0.1) * 0.53
    step = math.sqrt(0.1) * 2.0 ** -4                     # of the grid between 1/2 and 1 of the largest
    assert len(root.unique()) == 2
    # the mean of 102000 draws between neighbours: within 5 of its standard deviations
    assert abs(root.mean().item() - want) < 5 * step / 2 / math.sqrt(root.numel())
    b.load_state_dict(a.state_dict())
    a.step([g], lr=0.0, seed=8)
    b.step([g], lr=0.0, seed=9)
    assert not torch.equal(a.root.view(torch.uint8), b.root.view(torch.uint8)) and a.t == b.t == 2


def test_adamw_bad_gradients_and_tiny_states():
    p = torch.ones(1024, device="cuda")
    o = ops.AdamW([p], bits=8)
    g = torch.full((1024,), 1e-3, device="cuda")
    g[300] = float("nan")
    g[600] = float("inf")
    o.step([g], lr=0.1)
    m = decode(o.m, o.m_scale)
    assert m[1].isnan().all() and not m[2].isfinite().any() and m[[0, 3]].isfinite().all()
    assert p.isfinite().sum() == 1022
    q = torch.ones(512, device="cuda")
    o = ops.AdamW([q], bits=8)
    o.step([torch.full((512,), 1e-32, device="cuda")], lr=0.1)     # below what a scale can hold
    assert (o.m_scale == 0).all() and (o.root_scale == 0).all() and q.isfinite().all()
    o.step([torch.zeros(512, device="cuda")], lr=0.1)
    assert q.isfinite().all()


def test_adamw_many_tensors_strides_and_places():
    # more tensors than the small argument block holds, odd places, rows of a wider matrix
    g = gen(4)
    flat = randn(g, 70000)
    ps, at = [], 1
    for i in range(150):
        n = (i * 53) % 400 + (i % 3 == 0)
        ps.append(flat[at:at + n])
        at += n + (i % 4)
    wide = randn(g, 5, 1000)
    ps.append(wide[:, 3:900])
    start = [p.clone() for p in ps]
    keep = flat.clone(), wide.clone()
    copy = torch.zeros(5, 1001, dtype=HF, device="cuda")
    o = ops.AdamW(ps, decay=0.01, copies=[None] * 150 + [copy[:, 1:898]])
    gs = [randn(g, *p.shape, dtype=BF) for p in ps]
    o.step(gs, lr=0.1)
    for p, p0, gr in zip(ps, start, gs):
        want, _, _, step = ref_adamw(p0.double(), gr.double(), 0.0 * p0.double(), 0.0 * p0.double(), 1, 0.1, 0.01)
        assert ((p.double() - want).abs() <= 2.0 ** -20 * (step.abs() + want.abs())).all()
    assert torch.equal(copy[:, 1:898], wide[:, 3:900].to(HF)) and (copy[:, 0] == 0).all() and (copy[:, 898:] == 0).all()
    assert torch.equal(wide[:, :3], keep[1][:, :3]) and torch.equal(wide[:, 900:], keep[1][:, 900:])
    touched = torch.zeros(70000, dtype=torch.bool, device="cuda")
    for p in ps[:150]:
        s = p.storage_offset()
        touched[s:s + p.numel()] = True
    assert torch.equal(flat[~touched], keep[0][~touched])


def test_adamw_argument_blocks_of_thousands():
    ps = [torch.ones(3, device="cuda") for _ in range(4100)]
    o = ops.AdamW(ps)
    gs = [torch.full((3,), 1.0 if i % 2 else -1.0, device="cuda") for i in range(4100)]
    o.step(gs, lr=0.5)
    got = torch.stack(ps)
    assert (got[1::2] - 0.5).abs().max() < 1e-5 and (got[::2] - 1.5).abs().max() < 1e-5
