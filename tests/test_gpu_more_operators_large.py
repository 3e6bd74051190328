"""Tensors whose elements, or whose rows' distances, pass 32 bits."""
import math

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(lib):
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    yield
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("D", [4096, 4099])
def test_rows_beyond_32_bits(D):
    T, k, G = 70001, 8, 50                                   # 2.3e9 elements
    g = gen(1)
    s = ops.sort_by_group(torch.randint(-1, G, (T, k), generator=g, device="cuda", dtype=torch.int32), G)
    x = torch.randn(T, D, generator=g, device="cuda", dtype=BF)
    xs = ops.dispatch(x, s.place, s.offsets)
    n = int(s.offsets[-1])
    assert xs.numel() > 2 ** 31 and n < T * k
    for a in range(0, T * k, 1 << 17):
        src = s.source[a:a + (1 << 17)].long()
        want = torch.where((src < 0)[:, None], 0.0, x[(src // k).clamp(min=0)])
        assert torch.equal(xs[a:a + (1 << 17)], want)
    # each token's entries hold the token: sums of small whole numbers of it are exact in fp32
    w = torch.randint(0, 4, (T, k), generator=g, device="cuda").float()
    has = s.place >= 0
    out = ops.combine(xs, s.place, w, out_dtype=F)
    total = (w * has).sum(1, keepdim=True)
    assert (out - total * x.float()).abs().max() <= 2.0 ** -20 * 40 * 6
    dy, dw = ops.combine_backward(x, xs, s.place, w, s.offsets)
    dot = x.float().square().sum(1, keepdim=True)
    assert ((dw - dot * has).abs() <= 2.0 ** -24 * (D / 32 + 64) * dot).all()
    del out, xs
    last = s.place[T - 1][has[T - 1]].long()
    assert torch.equal(dy[last], (x[T - 1].float() * w[T - 1][has[T - 1]][:, None]).to(BF)) and (dy[n:] == 0).all()


def test_norm_beyond_32_bits():
    n = 2 ** 31 + 12345
    g = torch.full((n,), 2.0 ** -10, device="cuda", dtype=BF)
    g[-1] = 512.0
    want = math.sqrt((n - 1) * 2.0 ** -20 + 2.0 ** 18)
    r = ops.clip_gradients([g], 1.0)
    assert abs(r.norm.item() / want - 1) < 2e-6
    s = r.scale.item()
    assert g[-1].item() == torch.tensor(512 * r.scale.item()).to(BF).item()
    assert (g[:-1] == torch.tensor(2.0 ** -10 * s).to(BF).item()).all()


def test_logits_beyond_32_bits():
    wide = torch.zeros(40001, 60000, device="cuda", dtype=BF)
    z = wide[:, 59000:59064]
    z.copy_(torch.randn(40001, 64, generator=gen(2), device="cuda"))
    r = ops.route(z, 4)
    want = ops.route(z.contiguous(), 4)
    assert all(torch.equal(a, b) for a, b in zip(r, want))
    dw = torch.randn(40001, 4, generator=gen(3), device="cuda")
    d = ops.route_backward(dw, z, r.experts, r.weights, lse=r.lse, over="all")
    assert torch.equal(d, ops.route_backward(dw, z.contiguous(), r.experts, r.weights, lse=r.lse, over="all"))
    assert ops.route_backward(dw, z, r.experts, r.weights, lse=r.lse, over="all", out=z) is z and torch.equal(z, d)


def test_drafts_beyond_32_bits():
    B, K, V = 300, 7, 1000003                                # 2.4e9 logits
    g = gen(4)
    z = torch.empty(B, K + 1, V, device="cuda", dtype=BF)
    for b in range(B):
        z[b] = torch.randn(K + 1, V, generator=g, device="cuda")
    x = torch.randint(0, V, (B, K), generator=g, device="cuda", dtype=torch.int32)
    z.scatter_(2, torch.nn.functional.pad(x, (0, 1)).long()[..., None], 16.0)
    u = torch.rand(B, K, generator=g, device="cuda")
    noise = torch.empty(B, V, device="cuda").exponential_(generator=g)
    r = ops.verify_drafts(z, x, u, noise)
    # a draft has e^16 / (e^16 + 1000002 e^0.5) = 0.8434 of a row: all seven are accepted in 0.304 of the sequences, give or
    # take 5 times sqrt(0.304 * 0.696 / 300) = 0.0266
    assert abs((r.accepted == K).float().mean().item() - 0.304) <= 5 * 0.0266
    for at in (slice(0, 2), slice(B // 2, B // 2 + 1), slice(B - 2, B)):
        few = ops.verify_drafts(z[at].clone(), x[at].clone(), u[at].clone(), noise[at].clone())
        assert torch.equal(few.tokens, r.tokens[at]) and torch.equal(few.accepted, r.accepted[at])
        assert (few.logp - r.logp[at]).abs().max() <= 2.0 ** -17
        p = torch.softmax(z[at].double(), 2)
        ok = (u[at].double() < p[:, :K].gather(2, x[at].long()[..., None])[..., 0]).long().cumprod(1).sum(1)
        assert torch.equal(ok.int(), r.accepted[at])
