"""The operators at the edges of their domains, on the GPU: values, lengths and arguments where a formula
that holds elsewhere can fail."""
import math

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_gpu_operators import BF, F, HF, gen

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
