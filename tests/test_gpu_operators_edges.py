"""The operators at the edges of their domains, on the GPU: values, lengths and arguments where a formula
that holds elsewhere can fail."""
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
