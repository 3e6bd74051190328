"""Drafted tokens verified, on the GPU, against the rule in 64 bits, sequence by sequence."""
import math

import numpy as np
import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(B, K, V, dtype, probs, masked, temperature, seed, sure=True):
    g = gen(seed)
    z = torch.randn(B, K + 1, V, generator=g, device="cuda") * 2
    at = torch.randint(0, V, (B, K + 1, 1), generator=g, device="cuda")
    if sure:
        z.scatter_(2, at, math.log(V) + 3.0)
    ok = None
    if masked:
        ok = torch.rand(B, K + 1, V, generator=g, device="cuda") < 0.5
        ok.scatter_(2, at, True)
    d = (z[:, :K] + 0.8 * torch.randn(B, K, V, generator=g, device="cuda")) / temperature
    if masked:
        d = d.masked_fill(~ok[:, :K], -math.inf)
    q = torch.softmax(d, 2)
    if probs is None:
        x = q.argmax(2) if K else torch.zeros(B, 0, dtype=torch.long, device="cuda")
        q = None
    else:
        x = (q / torch.empty_like(q).exponential_(generator=g)).argmax(2) if K else torch.zeros(B, 0, dtype=torch.long, device="cuda")
        q = q.to(probs)
    x = torch.where(torch.rand(B, K, generator=g, device="cuda") < 0.1, -1, x)
    u = torch.rand(B, K, generator=g, device="cuda")
    noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    return z.to(dtype), x.int(), u, noise, q, ok


def want(z, x, u, noise, q=None, ok=None, temperature=1.0):
    z, x, u, noise = (a.double().cpu().numpy() for a in (z, x, u, noise))
    q = None if q is None else q.double().cpu().numpy()
    B, R, V = z.shape
    ok = np.ones(z.shape, bool) if ok is None else ok.cpu().numpy().astype(bool)
    tokens, accepted, logp = np.full((B, R), -1), np.zeros(B, int), np.zeros((B, R))
    far = np.ones((B, R))                                    # the tokens' distances to the largest logit
    with np.errstate(all="ignore"):
        for b in range(B):
            n = 0
            while True:
                in_ = ok[b, n] & ~(z[b, n] <= -1e30)
                s = np.where(in_, z[b, n] / temperature, -np.inf)
                bad = np.isnan(s).any() or (s == np.inf).any()
                m = s.max() if in_.any() else 0.0
                lse = m + np.log(np.exp(s - m).sum())
                p = np.zeros(V) if bad or not in_.any() else np.exp(s - lse)
                c = int(x[b, n]) if n < R - 1 else -1
                if c < 0:
                    rejected = False
                    break
                qc = 1.0 if q is None else q[b, n, c] if c < V else 0.0
                if not (c < V and u[b, n] * qc < p[c]):
                    rejected = True
                    break
                tokens[b, n], logp[b, n], far[b, n] = c, s[c] - lse, m - s[c]
                n += 1
            accepted[b] = n
            if bad:
                logp[b, n] = np.nan
                continue
            if not in_.any():
                logp[b, n] = -np.inf
                continue
            r = p
            if rejected:
                if q is None:
                    r = p.copy()
                    if c < V:
                        r[c] = 0.0
                else:
                    r = np.maximum(p - q[b, n], 0.0)
                if not (r > 0).any():
                    r = p
            t = int(np.argmax(np.where(r > 0, r / noise[b], -1.0)))
            tokens[b, n], logp[b, n], far[b, n] = t, s[t] - lse, m - s[t]
    return tokens, accepted, logp, far


def check(z, x, u, noise, q=None, ok=None, temperature=1.0):
    r = ops.verify_drafts(z, x, u, noise, draft_probs=q, temperature=temperature, allowed=ok)
    tokens, accepted, logp, far = want(z, x, u, noise, q, ok, temperature)
    assert r.tokens.dtype == r.accepted.dtype == torch.int32
    assert np.array_equal(r.accepted.cpu().numpy(), accepted)
    assert np.array_equal(r.tokens.cpu().numpy(), tokens)
    got = r.logp.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(logp)) and np.array_equal(np.isinf(got), np.isinf(logp))
    fin = np.isfinite(logp)
    # of the log sum: its terms' 2^-22 and arguments, weighted by themselves, and a chain of additions; of the difference
    # its rounding and the temperature's inverse's
    V = z.shape[2]
    tol = 2.0 ** -22 * (24 + V / 512 / 4 / 4 + far + np.abs(np.where(fin, logp, 0)))
    off = np.abs(got[fin] - logp[fin])
    assert (off <= tol[fin]).all(), off.max()
    return r


CASES = [(1, 4, 5), (3, 1, 100), (2, 3, 1001), (40, 5, 333), (1, 4, 33001), (5, 8, 9000), (200, 2, 1003), (7, 0, 4000), (1, 40, 50)]


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("probs", [F, BF, HF, None])
@pytest.mark.parametrize("B,K,V", CASES)
def test_verify(B, K, V, probs, dtype):
    for masked, temperature in ((False, 1.0), (True, 0.7)):
        z, x, u, noise, q, ok = make(B, K, V, dtype, probs, masked, temperature, B + K + V)
        r = check(z, x, u, noise, q, ok, temperature)
        check(z, x.long(), u, noise, q, ok, temperature)
        if ok is not None:                                   # the mask in the logits
            r2 = check(z.masked_fill(~ok, -math.inf), x, u, noise, q, None, temperature)
            assert torch.equal(r.tokens, r2.tokens)


@pytest.mark.parametrize("dtype", [F, BF, HF])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 9, 15, 17, 23, 33])
def test_few_classes(V, dtype):
    # rows that are all head and tail, from every alignment on
    for probs in (F, None):
        for masked in (False, True):
            z, x, u, noise, q, ok = make(9, 3, V, dtype, probs, masked, 1.0, V, sure=False)
            check(z, x, u, noise, q, ok)


def test_the_binding_and_the_host_module_agree():
    z, x, u, noise, q, ok = make(12, 3, 5000, BF, F, True, 0.9, 21)
    a = ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok, temperature=0.9)
    b = ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok, temperature=0.9, stream=torch.cuda.current_stream())
    assert all(torch.equal(p, r) for p, r in zip(a, b))


def test_flat_rows_and_a_token_from_given_noise():
    # nothing is sure: many classes share the probability
    for V in (10, 5000, 40000):
        z, x, u, noise, q, ok = make(30, 3, V, F, F, False, 1.3, V, sure=False)
        check(z, x, u, noise, q, ok, 1.3)
        check(z[:, :1], x[:, :0], u[:, :0], noise)
    # 20000 draws of one row have its probabilities
    p = torch.tensor([0.5, 0.25, 0.125, 0.125], device="cuda")
    n = 20000
    noise = torch.empty(n, 4, device="cuda").exponential_(generator=gen(3))
    none = torch.zeros(n, 0, device="cuda")
    t = ops.verify_drafts(p.log().expand(n, 1, 4), none.int(), none, noise).tokens[:, 0]
    share = torch.bincount(t, minlength=4) / n
    assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all()


def test_equal_scores_and_decisions_next_to_a_border():
    # equal r / noise: the lowest index; the sums are too close for 32 bits and are taken in 64
    V = 3000
    z = torch.zeros(2, 2, V, device="cuda")
    noise = torch.ones(2, V, device="cuda")
    noise[1, 7:] = 0.5
    x = torch.tensor([[-1], [-1]], dtype=torch.int32, device="cuda")
    r = check(z, x, torch.zeros(2, 1, device="cuda"), noise)
    assert r.tokens.tolist() == [[0, -1], [7, -1]]
    # u q against p: equal to 2^-24 of it
    g = gen(1)
    z = torch.randn(64, 2, 500, generator=g, device="cuda")
    x = z[:, :1].argmax(2).int()
    p = torch.softmax(z[:, 0].double(), 1).gather(1, x.long())
    u = p.float()
    noise = torch.empty(64, 500, device="cuda").exponential_(generator=g)
    step = torch.randint(-2, 3, (64, 1), generator=g, device="cuda")
    u = (u.view(torch.int32) + step).int().view(torch.float32)
    r = check(z, x, u, noise)
    assert 5 < r.accepted.sum() < 59
    # neighbouring noise
    noise = torch.full((8, 500), 0.75, device="cuda")
    noise[:, 1::3] = torch.nextafter(noise[:, 1::3], torch.ones([], device="cuda") * 0)
    check(torch.full((8, 1, 500), 2.5, device="cuda"), x[:8, :0], u[:8, :0], noise)


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("V,temperature", [(20011, 0.7), (3000, 1.0), (20011, 3.0)])
def test_borders_of_long_rows(V, temperature, dtype):
    # u is p's fp32 neighbours: the sum of thousands of exponentials has to be known to 2^-26 of it, and mostly far better
    g = gen(V)
    z = (torch.randn(48, 2, V, generator=g, device="cuda") * 2).to(dtype)
    x = z[:, :1].argmax(2).int()
    p = torch.softmax(z[:, 0].double() / temperature, 1).gather(1, x.long())
    u = (p.float().view(torch.int32) + torch.randint(-1, 2, (48, 1), generator=g, device="cuda")).int().view(torch.float32)
    noise = torch.empty(48, V, device="cuda").exponential_(generator=g)
    check(z, x, u, noise, None, None, temperature)
    q = torch.full((48, 1, V), 0.75, device="cuda")
    check(z, x, (p / 0.75).float(), noise, q, None, temperature)


def test_nothing_left_after_a_rejection():
    # q is at least p everywhere, and u says no: p is then drawn from
    z = torch.randn(6, 2, 40, generator=gen(2), device="cuda")
    q = (torch.softmax(z[:, :1], 2) * 2).contiguous()
    x = torch.randint(0, 40, (6, 1), generator=gen(3), device="cuda").int()
    u = torch.full((6, 1), 0.9, device="cuda")
    noise = torch.empty(6, 40, device="cuda").exponential_(generator=gen(4))
    assert (check(z, x, u, noise, q).accepted == 0).all()
    # one class alone, which was rejected
    ok = torch.zeros(40, dtype=torch.bool, device="cuda")
    ok[5] = True
    x[:] = 5
    u[:] = 1.0                                               # not below p = 1
    r = check(z, x, u, noise, None, ok.expand(6, 2, 40))
    assert (r.tokens[:, 0] == 5).all()
    # residuals of a few 2^-24, at classes of tiny probability
    z[:, 0, 3] = -60.0
    q = torch.softmax(z[:, :1].double(), 2).float()
    q[:, :, 3] = 0.0
    check(z, x, torch.full((6, 1), 0.99999994, device="cuda"), noise, q)


@pytest.mark.parametrize("dtype", [F, BF])
def test_rows_without_a_class_and_bad_rows(dtype):
    V = 700
    z, x, u, noise, q, _ = make(8, 3, V, dtype, F, False, 1.0, 5)
    u[:] = 0.0
    x[:] = torch.randint(0, V, (8, 3), generator=gen(1), device="cuda")
    z[0, 0], z[1, 2], z[2, 3] = -math.inf, torch.finfo(dtype).min, -2e30
    z[3, 1, 9], z[4, 0, 0], z[5, 3, V - 1] = math.nan, math.inf, math.nan
    x[6, 1] = V                                              # no class: rejected
    x[7, 0] = 2 ** 31 - 1
    r = check(z, x, u, noise, q)
    assert r.accepted.tolist() == [0, 2, 3, 1, 0, 3, 1, 0]
    assert r.logp[0, 0] == -math.inf and r.logp[2, 3] == -math.inf and r.logp[3, 1].isnan()
    check(z, x, u, noise, None)
    ok = torch.rand(8, 4, V, generator=gen(2), device="cuda") < 0.5
    ok[3, 1, 9] = False                                      # a NaN behind the mask is not seen
    ok[6] = False
    assert check(z, x, u, noise, q, ok).logp[3, 1].isfinite()
    check(z, x, u, noise, q, ok[0, 0].clone().expand(8, 4, V))
    r = ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok[1, 1].clone())
    assert torch.equal(r.tokens, ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok[1, 1].expand(8, 4, V)).tokens)


def test_temperatures_and_values_at_the_ends():
    for t in (1e-30, 1e-3, 50.0, 1e27):
        z, x, u, noise, q, _ = make(6, 2, 900, F, F, False, 1.0, 3)
        z = (z * 8).round() / 8
        check(z, x, u, noise, q, None, t)
    z = torch.full((2, 1, 300), -3e29, device="cuda")
    z[:, :, 5] = 3e38
    none = torch.zeros(2, 0, device="cuda")
    noise = torch.ones(2, 300, device="cuda")
    assert ops.verify_drafts(z, none.int(), none, noise).tokens.tolist() == [[5], [5]]


def test_strides():
    B, K, V = 5, 3, 1500
    z, x, u, noise, q, ok = make(B, K, V, BF, F, True, 1.0, 9)
    wide = torch.zeros(B, K + 3, V + 7, dtype=BF, device="cuda")
    wide[:, 1:K + 2, 3:V + 3] = z
    wq = torch.zeros(B, K + 1, V + 5, device="cuda")
    wq[:, :K, 1:V + 1] = q
    wn = torch.ones(B, V + 1, device="cuda")
    wn[:, 1:] = noise
    wo = torch.zeros(K + 1, B, V + 2, dtype=torch.uint8, device="cuda")
    wo[:, :, 1:V + 1] = ok.transpose(0, 1) * 3
    want_ = check(z, x, u, noise, q, ok)
    got = ops.verify_drafts(wide[:, 1:K + 2, 3:V + 3], x, u, wn[:, 1:], draft_probs=wq[:, :K, 1:V + 1],
                            allowed=wo[:, :, 1:V + 1].transpose(0, 1))
    assert torch.equal(got.tokens, want_.tokens) and torch.equal(got.accepted, want_.accepted)
    assert (got.logp - want_.logp).abs().max() <= 2.0 ** -18  # the vectors begin elsewhere: other orders of the sums
    empty = ops.verify_drafts(z[:0], x[:0], u[:0], noise[:0], draft_probs=q[:0])
    assert empty.tokens.shape == (0, K + 1) and empty.accepted.shape == (0,)


def test_captured_and_on_streams():
    z, x, u, noise, q, ok = make(9, 4, 8000, BF, F, False, 0.9, 2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    first = ops.verify_drafts(z, x, u, noise, draft_probs=q, temperature=0.9, stream=side)
    side.synchronize()
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            got.append(ops.verify_drafts(z, x, u, noise, draft_probs=q, temperature=0.9))
    for graph, r in zip(graphs, got):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(r, first))
    u.copy_(torch.rand(9, 4, generator=gen(11), device="cuda"))
    for graph in graphs:
        graph.replay()
    fresh = check(z, x, u, noise, q, None, 0.9)
    assert all(torch.equal(a, b) for r in got for a, b in zip(r, fresh))


@pytest.mark.parametrize("B,K,V", [(3, 15, 1), (5, 15, 2500), (7, 16, 2500), (4, 40, 333), (2, 70, 9), (1, 0, 8192), (1, 0, 8193),
                                   (2, 4, 8192), (2, 5, 8191), (63, 1, 9000), (64, 1, 9001), (64, 0, 16384), (64, 0, 16385),
                                   (64, 7, 16384), (65, 8, 16383), (512, 2, 257), (513, 2, 257), (1200, 1, 45)])
def test_next_to_the_limits_of_one_kernel(B, K, V):
    # A chain of a thread that shares a row with 31 others has V / 32 / 4 additions at most, 2500 classes: 20 of 2^-24, 5 steps of
    # 2^-22 (16384 classes, 2 warps of 16-bit vectors: 32 of 2^-24).  The others' 24 take 1 for the power, log2(V) / 2 <= 7
    # for the arguments, 3 at the end.
    for dtype, probs, masked in ((BF, F, True), (F, None, False), (HF, BF, False)):
        if V > 2500 and dtype == F and K > 5:
            continue
        check(*make(B, K, V, dtype, probs, masked, 1.0, B + K + V))


def test_a_batch_has_its_sequences_tokens():
    # 520 sequences take two kernels, 70 of them one with 512 threads each
    z, x, u, noise, q, ok = make(520, 3, 2001, BF, HF, True, 1.0, 77, sure=False)
    a = ops.verify_drafts(z, x, u, noise, draft_probs=q, allowed=ok)
    for i in range(0, 520, 70):
        b = ops.verify_drafts(*(t[i:i + 70] for t in (z, x, u, noise)), draft_probs=q[i:i + 70], allowed=ok[i:i + 70])
        assert torch.equal(a.tokens[i:i + 70], b.tokens) and torch.equal(a.accepted[i:i + 70], b.accepted)
        # each within 2^-22 (24 + 13 + |logp|), as above, of the same number
        assert ((a.logp[i:i + 70] - b.logp).abs() <= 2.0 ** -21 * (37 + b.logp.abs())).all()


@pytest.mark.parametrize("B,V", [(40, 1001), (600, 1001), (20, 20011)])
@pytest.mark.parametrize("dtype", [F, BF])
def test_a_large_class_that_the_draft_knew(dtype, B, V):
    # p = q but for its rounding at a class of p = 0.8 and little noise: its score's bound is above all others, its score is not
    g = gen(B + V)
    z = torch.randn(B, 2, V, generator=g, device="cuda")
    at = torch.randint(1, V, (B, 1), generator=g, device="cuda")
    z[:, 0].scatter_(1, at, math.log(V) + 1.9)
    z = z.to(dtype)
    p = torch.softmax(z[:, 0].double(), 1)
    q = (p * torch.rand(B, V, generator=g, device="cuda").double() * 2).scatter(1, at, p.gather(1, at))
    q[:, 0] = 1.0
    x = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    small = 10.0 ** (-9 + 6 * torch.rand(B, 1, generator=g, device="cuda"))
    r = check(z, x, torch.full((B, 1), 0.99, device="cuda"), noise.scatter(1, at, small), q.float()[:, None])
    assert r.accepted.eq(0).all()
    drawn = r.tokens[:, 0] == at[:, 0]
    assert drawn.any() and not drawn.all()
