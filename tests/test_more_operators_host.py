"""The host module and its build: what results hold, calls that are noted, a machine without a compiler for it."""
import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_operators_binding import BF, F, I32


@pytest.fixture
def noting(lib):
    host = ops._lib.host()
    host.pretend(True)
    yield host
    host.pretend(False)


def held(results):
    return max(t.untyped_storage().nbytes() for t in results), sum(-(-t.numel() * t.element_size() // 256) * 256 for t in results)


def test_results_hold_no_workspace(noting):
    # 136 KB of counts, 0.7 MB of sums and scores, a sum for each 2 KB
    r = noting.route(torch.zeros(3000, 200), 2, False, None)
    assert len(r) == 6 and held(r)[0] <= held(r)[1] + 8192
    r = noting.verify(torch.zeros(200, 6, 50), torch.zeros(200, 5, dtype=I32), torch.zeros(200, 5), torch.zeros(200, 50), None, 1.0, None)
    assert len(r) == 3 and held(r)[0] <= held(r)[1] + 8192
    r = noting.norm([torch.zeros(4, 3000, dtype=BF)] * 500, 1.0, 4, False)
    assert len(r) == 2 and held(r)[0] <= held(r)[1] + 8192 and r[0].dtype == F
    assert noting.pretend(True)[10] > 8192                   # (which is there all the same)
