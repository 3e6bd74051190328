"""Refusals of the operators: bad arguments come back as statuses from the C ABI before anything
touches the GPU, and as ValueError from the binding."""
import ctypes

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops

P = ctypes.c_void_p(1 << 12)      # an address that is never read
EINVAL, ENOMEM, EUNSUPPORTED = -1, -2, -6


def product(lib, **kw):
    a = dict(x=P, x_ld=64, w=P, w_ld=64, w_gs=4096, type=1, off=P, groups=2, rows=8, inner=64, outer=64,
             bias=None, bias_ld=0, relu=0, y=P, y_ld=64, y_type=1, ws=None, n=0)
    a.update(kw)
    return lib.hier_avg_grouped_product(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(type=0), EINVAL), (dict(type=3), EINVAL), (dict(y_type=2), EINVAL), (dict(groups=0), EINVAL),
    (dict(rows=-1), EINVAL), (dict(inner=0), EINVAL), (dict(outer=0), EINVAL), (dict(x_ld=63), EINVAL),
    (dict(w_ld=63), EINVAL), (dict(y_ld=63), EINVAL), (dict(x=None), EINVAL), (dict(off=None), EINVAL),
    (dict(y=None), EINVAL), (dict(n=-1), EINVAL), (dict(groups=1025), EUNSUPPORTED), (dict(x_ld=65), ENOMEM),
    (dict(w_gs=4097), ENOMEM), (dict(rows=0), 0), (dict(x=ctypes.c_void_p(4097)), EINVAL),
    (dict(rows=1 << 40), EINVAL)])
def test_product_refuses(lib, kw, status):
    assert product(lib, **kw) == status


def test_gradients_refuse(lib):
    dx = [P, 64, P, 64, 4096, 1, P, 2, 8, 64, 64, None, 0, P, 64, 1, None, 0, None]
    for at, v, status in ((0, None, EINVAL), (1, 3, EINVAL), (5, 0, EINVAL), (7, 2000, EUNSUPPORTED), (15, 2, EINVAL), (1, 66, ENOMEM)):
        a = list(dx)
        a[at] = v
        assert lib.hier_avg_grouped_product_dx(*a) == status, (at, v)
    a = list(dx)
    a[11], a[12] = P, 10                                    # rows of h that overlap
    assert lib.hier_avg_grouped_product_dx(*a) == EINVAL
    dw = [P, 64, P, 64, 1, P, 2, 8, 64, 64, P, 64, 4096, 1, None, 0, None, 0, None]
    for at, v, status in ((0, None, EINVAL), (4, 0, EINVAL), (6, 2000, EUNSUPPORTED), (10, None, EINVAL), (11, 5, EINVAL), (13, 2, EINVAL), (3, 65, ENOMEM)):
        a = list(dw)
        a[at] = v
        assert lib.hier_avg_grouped_product_dw(*a) == status, (at, v)


def test_workspace(lib):
    n = ctypes.c_int64(-1)
    f = lib.hier_avg_grouped_product_workspace
    assert f(0, P, 64, P, 64, 4096, 2, 8, 64, 64, ctypes.byref(n)) == 0 and n.value == 0
    assert f(0, P, 65, P, 64, 4096, 2, 8, 64, 64, ctypes.byref(n)) == 0 and n.value == 8 * 64 * 2
    assert f(2, P, 64, P, 70, 0, 2, 8, 64, 64, ctypes.byref(n)) == 0 and n.value >= 8 * 64 * 2
    assert f(3, P, 64, P, 64, 0, 2, 8, 64, 64, ctypes.byref(n)) == EINVAL
    assert f(0, P, 64, P, 64, 0, 2, 8, 64, 64, None) == EINVAL


def test_workspace_of_parts(lib):
    # few tiles over many rows: the weights' gradient's parts need room
    n = ctypes.c_int64(-1)
    assert lib.hier_avg_grouped_product_workspace(2, P, 64, P, 64, 0, 1, 8192, 64, 64, ctypes.byref(n)) == 0
    assert n.value >= 2 * 64 * 64 * 4
    dw = [P, 64, P, 64, 1, P, 1, 8192, 64, 64, P, 64, 4096, 1, None, 0, P, n.value - 1, None]
    assert lib.hier_avg_grouped_product_dw(*dw) == ENOMEM
    assert lib.hier_avg_grouped_product_workspace(2, P, 64, P, 64, 0, 1000, 1 << 24, 64, 64, ctypes.byref(n)) == 0
    assert n.value == 0


def test_workspace_counted_here(lib):
    # the Python side counts the copies itself; the library refuses less than it needs
    import random

    from paper_1903_05133_gb300 import operators as ops

    class Fake:                                             # a tensor as far as its address goes
        device = "cpu"

        def __init__(self, address):
            self.data_ptr = lambda: address

    rng = random.Random(5)
    n = ctypes.c_int64()
    for _ in range(2000):
        op, groups, rows = rng.randrange(3), rng.choice((1, 2, 9)), rng.randrange(1, 500)
        inner, outer = rng.randrange(1, 200), rng.randrange(1, 200)
        inner, outer = (v * 8 if rng.random() < 0.5 else v for v in (inner, outer))
        a, b = (Fake(P.value + rng.choice((0, 0, 0, 2, 8, 16))) for _ in range(2))
        pad = lambda v: v + rng.choice((0, 0, 1, 8))  # noqa: E731
        a_ld, b_ld = pad(inner if op == 0 else outer), pad(inner)
        b_gs = 0 if op == 2 else rng.choice((0, outer * b_ld, outer * b_ld + 3, outer * b_ld + 8))
        assert lib.hier_avg_grouped_product_workspace(op, a.data_ptr(), a_ld, b.data_ptr(), b_ld, b_gs, groups, rows, inner, outer,
                                                      ctypes.byref(n)) == 0
        assert ops._workspace(lib, op, a, a_ld, b, b_ld, b_gs, groups, rows, inner, outer)[2] == n.value


def test_logprobs_refuse(lib):
    fwd = [P, 1, 4, 100, 100, P, 4, None, 0, 1.0, 3, P, P, P, P, P, None]
    for at, v, status in ((0, None, EINVAL), (1, 3, EINVAL), (2, -1, EINVAL), (3, 0, EINVAL), (4, 99, EINVAL), (5, None, EINVAL),
                          (6, 2, EINVAL), (8, 50, EINVAL), (9, 0.0, EINVAL), (9, float("nan"), EINVAL), (10, -1, EINVAL),
                          (10, 33, EUNSUPPORTED), (11, None, EINVAL), (14, None, EINVAL), (2, 0, 0), (2, 1 << 31, EUNSUPPORTED)):
        a = list(fwd)
        a[at] = v
        assert lib.hier_avg_token_logprobs(*a) == status, (at, v)
    bwd = [P, 1, 4, 100, 100, P, 4, None, 0, 1.0, P, P, P, P, P, 100, None]
    for at, v, status in ((0, None, EINVAL), (10, None, EINVAL), (11, None, EINVAL), (12, None, EINVAL), (14, None, EINVAL),
                          (15, 99, EINVAL), (2, 0, 0), (2, 1 << 40, EUNSUPPORTED)):
        a = list(bwd)
        a[at] = v
        assert lib.hier_avg_token_logprobs_backward(*a) == status, (at, v)


def create(lib, bits=8, tensors=1, n=(1000,), tensor=(0,), decay=(0.0,), offset=(0,)):
    h = ctypes.c_void_p()
    k = len(n)
    rc = lib.hier_avg_adamw_create(bits, tensors, k, (ctypes.c_int * k)(*tensor), (ctypes.c_void_p * k)(*[4096] * k), None, 0,
                                   (ctypes.c_int64 * k)(*n), (ctypes.c_int64 * k)(*offset), (ctypes.c_float * k)(*decay),
                                   ctypes.byref(h))
    return rc, h


def test_adamw_refuses(lib):
    for kw in (dict(bits=16), dict(tensors=0), dict(n=(-1,)), dict(tensor=(1,)), dict(tensor=(-1,)), dict(offset=(-1,)),
               dict(decay=(float("nan"),)), dict(n=(1, 1), tensor=(1, 0), decay=(0, 0), offset=(0, 0), tensors=2)):
        rc, h = create(lib, **kw)
        assert rc == EINVAL and not h.value, kw
    rc, h = create(lib, n=(1000, 1, 256), tensor=(0, 0, 2), decay=(0, 0, 0), offset=(0, 1000, 0), tensors=3)
    assert rc == 0
    e, b = ctypes.c_int64(), ctypes.c_int64()
    assert lib.hier_avg_adamw_sizes(h, ctypes.byref(e), ctypes.byref(b)) == 0 and e.value == 1024 + 256 + 256 and b.value > 0
    g = (ctypes.c_void_p * 3)(4096, None, 4096)
    step = lambda lr=0.1, b1=0.9, b2=0.99, eps=1e-8, t=1, kind=0: lib.hier_avg_adamw_step(  # noqa: E731
        h, g, kind, lr, b1, b2, eps, t, None, 0, None)
    for kw in (dict(lr=float("inf")), dict(b1=1.0), dict(b2=-0.1), dict(eps=0.0), dict(t=0), dict(kind=3)):
        assert step(**kw) == EINVAL, kw
    assert step() == -4                                     # HA_ESTATE: not bound
    assert lib.hier_avg_adamw_bind(h, P, b.value - 1, P, P, P, P, None) == ENOMEM
    assert lib.hier_avg_adamw_bind(h, P, b.value, P, P, None, P, None) == EINVAL
    lib.hier_avg_adamw_destroy(h)
    lib.hier_avg_adamw_destroy(None)


def test_binding_refuses(lib):
    t = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        ops.grouped_product(t, t[None], torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        ops.token_logprobs(t, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="CUDA"):
        ops.AdamW([torch.zeros(4)])
    with pytest.raises(ValueError, match="bits"):
        ops.AdamW([torch.zeros(4)], bits=4)
