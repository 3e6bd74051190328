"""What the routing, row, norm and draft operators refuse: by status from the C ABI, and by ValueError from
the binding, on stand-ins for CUDA tensors.  No address is read here."""
import ctypes

import pytest
import torch

from paper_1903_05133_gb300 import operators as ops
from test_operators_abi import EINVAL, ENOMEM, EUNSUPPORTED, P
from test_operators_binding import BF, BOOL, F, HF, I32, Calls, Guard, Stand, Stream

ODD = ctypes.c_void_p(4097)
FAR = 1 << 40


def refuses(call, good, cases):
    for at, v, status in cases:
        a = list(good)
        a[at] = v
        assert call(*a) == status, (at, v)


def test_sort_workspace(lib):
    n = ctypes.c_int64(-1)
    b = ctypes.byref(n)
    refuses(lib.hier_avg_sort_workspace, [1000, 8, 64, b], (
        (0, -1, EINVAL), (1, 0, EINVAL), (2, 0, EINVAL), (3, None, EINVAL), (1, 33, EUNSUPPORTED), (2, 1025, EUNSUPPORTED),
        (0, 1 << 28, EUNSUPPORTED), (0, FAR, EUNSUPPORTED)))
    # the binding knows without asking where nothing is needed, and how much is enough
    for rows in (0, 1, 31, 32, 33, 64, 256, 2048, 4863, 4864, 4865, 10000, 16384, 99999, 1 << 20, 1 << 22):
        for k in (1, 2, 8, 31, 32):
            assert lib.hier_avg_sort_workspace(rows, k, 64, b) == 0
            assert (n.value == 0) == (rows <= ops._ONE_ROWS and rows * k <= ops._ONE_ENTRIES), (rows, k)
            assert n.value <= ops._sort_bytes(lib, rows, k, 64) and (n.value or not ops._sort_bytes(lib, rows, k, 64))
    # any number of rows has chunks whose entries' ranks fit
    for rows, k in ((1 << 30, 1), (1 << 26, 31), ((1 << 31) - 1, 1)):
        assert lib.hier_avg_sort_workspace(rows, k, 1024, b) == 0 and n.value < 1 << 26


def test_route_refuses(lib):
    good = [P, 0, 8, 64, 64, 6, 0, None, 0, P, P, P, P, P, P, None, 0, None]
    refuses(lib.hier_avg_route, good, (
        (0, None, EINVAL), (0, ODD, EINVAL), (1, 3, EINVAL), (1, -1, EINVAL), (2, -1, EINVAL), (3, 0, EINVAL), (4, 63, EINVAL),
        (5, 0, EINVAL), (5, 65, EINVAL), (5, 33, EUNSUPPORTED), (8, 1, EINVAL), (9, None, EINVAL), (10, None, EINVAL),
        (11, None, EINVAL), (12, None, EINVAL), (13, None, EINVAL), (14, None, EINVAL), (16, -1, EINVAL), (2, 300, ENOMEM),
        (2, FAR, EUNSUPPORTED)))
    a = list(good)
    a[3], a[4], a[7], a[8] = 64, 64, P, 17                  # 1088 groups
    assert lib.hier_avg_route(*a) == EUNSUPPORTED
    a[8] = 0
    assert lib.hier_avg_route(*a) == EINVAL
    a[3], a[4], a[7], a[8] = 1025, 1025, None, 0
    assert lib.hier_avg_route(*a) == EUNSUPPORTED


def test_sort_and_route_backward_refuse(lib):
    refuses(lib.hier_avg_sort_by_group, [P, 8, 2, 10, P, P, P, None, 0, None], (
        (0, None, EINVAL), (1, -1, EINVAL), (2, 0, EINVAL), (3, 0, EINVAL), (4, None, EINVAL), (5, None, EINVAL), (6, None, EINVAL),
        (8, -1, EINVAL), (7, ODD, EINVAL), (2, 33, EUNSUPPORTED), (3, 1025, EUNSUPPORTED), (1, 2000, ENOMEM), (1, FAR, EUNSUPPORTED)))
    good = [P, P, 0, 8, 64, 64, 6, 1, P, P, P, P, 64, None]
    refuses(lib.hier_avg_route_backward, good, (
        (0, None, EINVAL), (1, None, EINVAL), (1, ODD, EINVAL), (2, 4, EINVAL), (3, -1, EINVAL), (4, 0, EINVAL), (5, 63, EINVAL),
        (6, 0, EINVAL), (6, 65, EINVAL), (8, None, EINVAL), (9, None, EINVAL), (10, None, EINVAL), (11, None, EINVAL),
        (11, ODD, EINVAL), (12, 63, EINVAL), (3, 0, 0), (3, FAR, EUNSUPPORTED)))
    a = list(good)
    a[7], a[1], a[10], a[3] = 0, None, None, 0              # over the chosen neither logits nor lse are read
    assert lib.hier_avg_route_backward(*a) == 0


def test_rows_refuse(lib):
    refuses(lib.hier_avg_dispatch, [P, 1, 8, 64, 64, P, 2, P, 4, P, 64, None], (
        (0, None, EINVAL), (0, ODD, EINVAL), (1, 3, EINVAL), (2, -1, EINVAL), (3, 0, EINVAL), (4, 63, EINVAL), (5, None, EINVAL),
        (6, 0, EINVAL), (7, None, EINVAL), (8, 0, EINVAL), (9, None, EINVAL), (9, ODD, EINVAL), (10, 63, EINVAL), (2, 0, 0),
        (2, 1 << 30, EUNSUPPORTED), (2, FAR, EUNSUPPORTED)))
    refuses(lib.hier_avg_combine, [P, 1, 8, 64, 64, P, 2, P, P, 64, 1, None], (
        (0, None, EINVAL), (0, ODD, EINVAL), (1, 3, EINVAL), (2, -1, EINVAL), (3, 0, EINVAL), (4, 63, EINVAL), (5, None, EINVAL),
        (6, 0, EINVAL), (8, None, EINVAL), (9, 63, EINVAL), (10, 2, EINVAL), (2, 0, 0), (2, FAR, EUNSUPPORTED)))
    refuses(lib.hier_avg_combine_backward, [P, 1, 64, P, 1, 8, 64, 64, P, 2, P, P, 4, P, 64, P, None], (
        (0, None, EINVAL), (1, 2, EINVAL), (2, 63, EINVAL), (3, None, EINVAL), (4, 3, EINVAL), (5, -1, EINVAL), (6, 0, EINVAL),
        (7, 63, EINVAL), (8, None, EINVAL), (9, 0, EINVAL), (10, None, EINVAL), (11, None, EINVAL), (12, 0, EINVAL),
        (13, None, EINVAL), (13, ODD, EINVAL), (14, 63, EINVAL), (15, None, EINVAL), (5, 0, 0), (5, FAR, EUNSUPPORTED)))


def arrays(sizes, types=None, address=None):
    n = len(sizes)
    return ((ctypes.c_void_p * n)(*(address or [4096 + i * 65536 for i in range(n)])), (ctypes.c_int * n)(*(types or [0] * n)),
            (ctypes.c_int64 * n)(*sizes))


def test_grad_norm_refuses(lib):
    g, t, n = arrays((100, 50, 0))
    b = ctypes.c_int64(-1)
    size = lambda *a: lib.hier_avg_grad_norm_workspace(*a, ctypes.byref(b))  # noqa: E731
    assert size(3, t, n, 1) == 0 and b.value == 16 and size(3, t, n, 50) == 0 and b.value == 800
    assert size(0, t, n, 1) == size(3, None, n, 1) == size(3, t, None, 1) == size(3, t, n, 0) == size(3, t, n, 7) == EINVAL
    assert size(3, (ctypes.c_int * 3)(0, 3, 0), n, 1) == size(3, t, (ctypes.c_int64 * 3)(1, -1, 0), 1) == EINVAL
    assert size(1, t, (ctypes.c_int64 * 1)(1 << 50), 1) == size(44801, t, n, 1) == EUNSUPPORTED
    good = [3, g, t, n, 1, 1.0, 1, P, P, P, 16, None]
    refuses(lib.hier_avg_grad_norm, good, (
        (0, 0, EINVAL), (1, None, EINVAL), (4, 0, EINVAL), (5, -1.0, EINVAL), (5, float("nan"), EINVAL), (5, float("inf"), EINVAL),
        (7, None, EINVAL), (8, None, EINVAL), (9, None, ENOMEM), (9, ctypes.c_void_p(4100), EINVAL), (10, 15, ENOMEM),
        (1, arrays((100, 50, 0), address=[4096, None, None])[0], EINVAL), (1, arrays((100, 50, 0), address=[4096, 8194, 1])[0], EINVAL),
        # tensors that share memory are not clipped, in whatever order they come
        (1, arrays((100, 50, 0), address=[4096, 4492, 1])[0], EINVAL), (1, arrays((100, 50, 0), address=[4096, 3900, 1])[0], EINVAL),
        (1, arrays((100, 50, 0), address=[4096, 4096, 1])[0], EINVAL)))


def test_verify_refuses(lib):
    b = ctypes.c_int64(-1)
    assert lib.hier_avg_verify_workspace(3, 4, ctypes.byref(b)) == 0 and b.value == 3 * (272 * 5 + 2052)   # as the binding counts it
    assert lib.hier_avg_verify_workspace(3, -1, ctypes.byref(b)) == lib.hier_avg_verify_workspace(-1, 4, ctypes.byref(b)) == EINVAL
    assert lib.hier_avg_verify_workspace(3, 2 ** 31 - 1, ctypes.byref(b)) == EUNSUPPORTED
    assert lib.hier_avg_verify_workspace(1 << 24, 0, ctypes.byref(b)) == lib.hier_avg_verify_workspace(1 << 20, 100, ctypes.byref(b)) == EUNSUPPORTED
    good = [P, 1, 3, 4, 100, 500, 100, P, 4, P, P, 100, P, 0, 400, 100, P, 500, 100, 1.0, P, P, P, P, 3 * 3412, None]
    cases = [(0, None, EINVAL), (0, ODD, EINVAL), (1, 3, EINVAL), (2, -1, EINVAL), (3, -1, EINVAL), (4, 0, EINVAL), (5, -1, EINVAL),
             (4, 2 ** 31 - 1, EINVAL), (6, -1, EINVAL), (7, None, EINVAL), (8, 2, EINVAL), (9, None, EINVAL), (10, None, EINVAL),
             (11, -1, EINVAL), (12, ODD, EINVAL), (13, 3, EINVAL), (14, -1, EINVAL), (15, -1, EINVAL), (17, -1, EINVAL),
             (18, -1, EINVAL), (20, None, EINVAL), (21, None, EINVAL), (22, None, EINVAL), (23, None, ENOMEM),
             (23, ctypes.c_void_p(4100), EINVAL), (24, 3 * 3411, ENOMEM), (2, 0, 0), (2, 1 << 26, EUNSUPPORTED)]
    cases += [(19, t, EINVAL) for t in (0.0, -1.0, 2.0 ** -127, 1.1e27, float("nan"), float("inf"))]
    refuses(lib.hier_avg_verify_drafts, good, cases)


# ---------------------------------------------------------------------- the binding
@pytest.fixture
def gpus(monkeypatch):
    """GPU 0 is current, the current stream of GPU d is 100 + d; results are stand-ins."""
    ops._lib.host()
    now = [0]
    calls = Calls(now)
    made = []

    def empties(like, *specs):
        kinds = (F, BF, HF, I32, torch.uint8)
        made.append((now[0], [s for s in specs]))
        return tuple(Stand(kinds[s[0]], s[1:], address=(1 << 40) + i * (1 << 30), gpu=like.get_device()) for i, s in enumerate(specs))
    monkeypatch.setattr(ops._lib, "load", lambda: calls)
    monkeypatch.setattr(ops, "_empties", empties)
    monkeypatch.setattr(ops, "_sort_bytes", lambda lib, rows, k, groups: 0)
    monkeypatch.setattr(ops, "_CURRENT", lambda: now[0])
    monkeypatch.setattr(ops, "_RAW_STREAM", lambda d: 100 + d)
    monkeypatch.setattr(torch.cuda, "device", lambda d: Guard(now, d))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: Guard(now, s.device_index))
    return now, calls, made


def every_call():
    T, k, E, D, G, B, K, V = 6, 2, 10, 24, 10, 3, 4, 50
    at = iter(range(1 << 20, 1 << 34, 1 << 20))

    def tensors(gpu):
        S = lambda name, dtype, shape: Stand(dtype, shape, address=next(at), gpu=gpu(name))  # noqa: E731
        off = lambda: S("offsets", I32, (G + 1,))  # noqa: E731
        place = lambda: S("place", I32, (T, k))  # noqa: E731
        w = lambda name="weights": S(name, F, (T, k))  # noqa: E731
        return {
            "route": lambda **q: ops.route(S("logits", BF, (T, E)), k, learners=S("learners", I32, (4,)), **q),
            "route_backward": lambda **q: ops.route_backward(
                w("dweights"), S("logits", BF, (T, E)), S("experts", I32, (T, k)), w(), lse=S("lse", F, (T,)), over="all",
                out=S("out", BF, (T, E)), **q),
            "sort_by_group": lambda **q: ops.sort_by_group(S("group", I32, (T, k)), G, **q),
            "dispatch": lambda **q: ops.dispatch(S("x", BF, (T, D)), place(), off(), out=S("out", BF, (T * k, D)), **q),
            "combine": lambda **q: ops.combine(S("y", BF, (T * k, D)), place(), w(), out=S("out", F, (T, D)), **q),
            "combine_backward": lambda **q: ops.combine_backward(
                S("dout", F, (T, D)), S("y", BF, (T * k, D)), place(), w(), off(), out=S("out", BF, (T * k, D)), **q),
            "verify_drafts": lambda **q: ops.verify_drafts(
                S("logits", BF, (B, K + 1, V)), S("drafts", I32, (B, K)), S("uniform", F, (B, K)), S("noise", F, (B, V)),
                draft_probs=S("draft_probs", HF, (B, K, V)), allowed=S("allowed", BOOL, (B, K + 1, V)), **q)}
    return tensors


NAMES = {"route": ("logits", "learners"), "route_backward": ("dweights", "logits", "experts", "weights", "lse", "out"),
         "sort_by_group": ("group",), "dispatch": ("x", "place", "offsets", "out"), "combine": ("y", "place", "weights", "out"),
         "combine_backward": ("dout", "y", "place", "weights", "offsets", "out"),
         "verify_drafts": ("logits", "drafts", "uniform", "noise", "draft_probs", "allowed")}


def test_calls_run_on_their_tensors_gpu(gpus):
    now, calls, made = gpus
    for gpu in (0, 1):
        for name, call in every_call()(lambda _: gpu).items():
            for kw, stream in (({}, 100 + gpu), ({"stream": Stream(gpu, 7)}, 7)):
                calls.made.clear()
                made.clear()
                call(**kw)
                assert calls.made == [("hier_avg_" + name, gpu, stream)] and now == [0], name
                assert all(d == gpu for d, _ in made)        # the results are made there, on the stream
            calls.made.clear()
            with pytest.raises(ValueError, match="stream"):
                call(stream=Stream(1 - gpu, 7))
            assert not calls.made


def test_tensors_of_two_gpus_are_refused(gpus):
    _, calls, _ = gpus
    for name, tensors in NAMES.items():
        for one in tensors if len(tensors) > 1 else ():
            with pytest.raises(ValueError, match="GPU"):
                every_call()(lambda n: int(n == one))[name]()
    assert not calls.made


ROOM = iter(range(1 << 20, 1 << 40, 1 << 20))


def S(dtype, shape, strides=None, address=None):
    return Stand(dtype, shape, strides, next(ROOM) if address is None else address)


def test_arguments_are_refused(gpus):
    T, k, E, D, B, K, V = 6, 2, 10, 24, 3, 4, 50
    z, e, w, off, place = S(BF, (T, E)), S(I32, (T, k)), S(F, (T, k)), S(I32, (E + 1,)), S(I32, (T, k))
    x, y = S(BF, (T, D)), S(BF, (T * k, D))
    lse = S(F, (T,))
    lz, d, u, no, q, ok = (S(BF, (B, K + 1, V)), S(I32, (B, K)), S(F, (B, K)), S(F, (B, V)), S(F, (B, K, V)), S(BOOL, (B, K + 1, V)))
    bad = [
        lambda: ops.route(z, 0), lambda: ops.route(z, 11), lambda: ops.route(S(BF, (T, 100)), 33), lambda: ops.route(z, 2, over="both"),
        lambda: ops.route(S(torch.float64, (T, E)), 2), lambda: ops.route(S(BF, (T, E), (5, 1)), 2),
        lambda: ops.route(S(BF, (T, E), (1, T)), 2), lambda: ops.route(S(BF, (T,)), 2), lambda: ops.route(S(BF, (T, 1025)), 2),
        lambda: ops.route(z, 2, learners=S(I32, (105,))), lambda: ops.route(z, 2, learners=S(torch.int64, (3,))),
        lambda: ops.route(z, 2, learners=S(I32, (1,))),
        lambda: ops.route_backward(w, z, S(I32, (T,)), w), lambda: ops.route_backward(w, z, S(torch.int64, (T, k)), w),
        lambda: ops.route_backward(w, z, e, w, over="all"), lambda: ops.route_backward(S(F, (T, 3)), z, e, w),
        lambda: ops.route_backward(w, z, e, S(F, (T, k), (1, T))), lambda: ops.route_backward(w, z, e, w, lse=S(F, (T + 1,)), over="all"),
        lambda: ops.route_backward(w, z, e, w, out=S(F, (T, E))), lambda: ops.route_backward(w, z, e, w, out=S(BF, (T, E), address=z.address + 2)),
        lambda: ops.route_backward(S(F, (T, 40)), S(BF, (T, 50)), S(I32, (T, 40)), S(F, (T, 40))),
        lambda: ops.sort_by_group(e, 0), lambda: ops.sort_by_group(e, 1025), lambda: ops.sort_by_group(S(I32, (T, 33)), 4),
        lambda: ops.sort_by_group(S(I32, (T,)), 4), lambda: ops.sort_by_group(S(torch.int64, (T, k)), 4),
        lambda: ops.sort_by_group(S(I32, (T, k), (4, 1)), 4),
        lambda: ops.dispatch(S(BF, (T + 1, D)), place, off), lambda: ops.dispatch(x, S(torch.int64, (T, k)), off),
        lambda: ops.dispatch(x, S(I32, (T, k), (3, 1)), off), lambda: ops.dispatch(x, place, S(F, (E + 1,))),
        lambda: ops.dispatch(x, place, off, out=S(BF, (T, D))), lambda: ops.dispatch(x, place, off, out=S(BF, (T * k, D), address=x.address)),
        lambda: ops.dispatch(S(BF, (T, D), (20, 1)), place, off), lambda: ops.dispatch(x, S(I32, (T, 0)), off),
        lambda: ops.combine(x, place, w), lambda: ops.combine(y, place, S(F, (T, 3))), lambda: ops.combine(y, place, S(BF, (T, k))),
        lambda: ops.combine(y, place, None),
        lambda: ops.combine(y, place, w, out_dtype=HF), lambda: ops.combine(S(F, (T * k, D)), place, w, out_dtype=BF),
        lambda: ops.combine(y, place, w, out=S(F, (T, D), address=y.address)), lambda: ops.dispatch_backward(x, place),
        lambda: ops.dispatch_backward(y, place, out_dtype=HF),
        lambda: ops.combine_backward(x, S(BF, (T, D)), place, w, off), lambda: ops.combine_backward(S(HF, (T, D)), y, place, w, off),
        lambda: ops.combine_backward(S(F, (T, D + 1)), y, place, w, off), lambda: ops.combine_backward(x, y, place, S(F, (T, 1)), off),
        lambda: ops.combine_backward(x, y, place, w, S(I32, (1,))), lambda: ops.combine_backward(x, y, place, w, off, out=S(F, (T * k, D))),
        lambda: ops.combine_backward(x, y, place, w, off, out=S(BF, (T * k, D), address=y.address)),
        lambda: ops.verify_drafts(S(BF, (B, V)), d, u, no), lambda: ops.verify_drafts(S(BF, (B, K + 1, V), (V * 5, V, 2)), d, u, no),
        lambda: ops.verify_drafts(S(BF, (B, 0, V)), d, u, no), lambda: ops.verify_drafts(lz, S(I32, (B, K + 1)), u, no),
        lambda: ops.verify_drafts(lz, S(F, (B, K)), u, no), lambda: ops.verify_drafts(lz, S(I32, (B, K), (5, 1)), u, no),
        lambda: ops.verify_drafts(lz, d, S(BF, (B, K)), no), lambda: ops.verify_drafts(lz, d, u, S(F, (B, V + 1))),
        lambda: ops.verify_drafts(lz, d, u, S(HF, (B, V))), lambda: ops.verify_drafts(lz, d, u, no, draft_probs=S(F, (B, K + 1, V))),
        lambda: ops.verify_drafts(lz, d, u, no, draft_probs=S(F, (B, K, V), (K * V, 1, K))),
        lambda: ops.verify_drafts(lz, d, u, no, allowed=S(BOOL, (V + 1,))), lambda: ops.verify_drafts(lz, d, u, no, allowed=S(F, (V,))),
        lambda: ops.verify_drafts(lz, d, u, no, allowed=S(BOOL, (B, V))),
        *[lambda t=t: ops.verify_drafts(lz, d, u, no, temperature=t) for t in (0.0, -1.0, float("nan"), float("inf"), 1e28, 1e-38)]]
    _, calls, _ = gpus
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"case {i} went through")
    assert not calls.made
    # and what is allowed goes through
    ops.route(z, 10), ops.route_backward(w, z, e, w), ops.route_backward(w, z, e, w, lse=lse, over="all", out=z)
    ops.verify_drafts(lz, d, u, no, q, 0.5, ok), ops.verify_drafts(lz, d, u, no, allowed=S(BOOL, (V,)))
    ops.verify_drafts(lz, d, u, no, allowed=S(BOOL, (B, K + 1, V), (0, 0, 1)))
    ops.verify_drafts(S(BF, (B, 1, V)), S(I32, (B, 0)), S(F, (B, 0)), no, draft_probs=S(F, (B, 0, V)))
    ops.combine(y, place, w, out_dtype=F), ops.dispatch_backward(y, place, out_dtype=F), ops.combine_backward(S(F, (T, D)), y, place, w, off)


def test_gradients_that_are_refused():
    cpu = torch.zeros(4)
    for bad, match in (([], "empty"), ([cpu], "CUDA"), ([cpu, 3], "CUDA"), ([None], "CUDA")):
        for call in (lambda: ops.grad_norm(bad, 1.0), lambda: ops.clip_gradients(bad, 1.0)):
            with pytest.raises(ValueError, match=match):
                call()
    with pytest.raises(ValueError, match="max_norm"):
        ops.clip_gradients([cpu], None)


def test_gradients_facts(lib):
    from paper_1903_05133_gb300 import _lib
    facts = _lib.host().facts
    assert facts([])[:3] == (b"", b"", b"") and facts((torch.zeros(3),))[3] == -1 and facts([7])[3] == -4
    with pytest.raises(TypeError):
        facts(3)


def test_results_made_together(lib):
    from paper_1903_05133_gb300 import _lib
    empties, like = _lib.host().empties, torch.zeros(1)
    a, b, c, d = empties(like, (0, 3, 5), (3, 7), (1, 0, 4), (4,))
    assert (a.dtype, b.dtype, c.dtype, d.dtype) == (F, I32, BF, torch.uint8)
    assert (tuple(a.shape), tuple(b.shape), tuple(c.shape), tuple(d.shape)) == ((3, 5), (7,), (0, 4), ())
    assert a.is_contiguous() and a.untyped_storage().data_ptr() == b.untyped_storage().data_ptr() and a.data_ptr() + 256 == b.data_ptr()
    a.fill_(1.5), b.fill_(2), d.fill_(3)
    assert (a == 1.5).all() and (b == 2).all() and d == 3 and a._version == 1 and b._version == 1
    big, small = empties(like, (0, 1 << 21), (0, 4))         # beyond 4 MB each has its own memory
    assert big.untyped_storage().nbytes() == 1 << 23 and small.untyped_storage().nbytes() == 16
    with torch.inference_mode():
        assert empties(like, (0, 2))[0].is_inference()
    for bad in ((), (3,), (like, (5, 1)), (like, (0, -1)), (like, [0, 1]), (like, (0, 1, 1, 1, 1)), (like, ("a",)), (like, ()),
                (like,) * 1 + ((0, 1),) * 16):
        with pytest.raises((TypeError, ValueError)):
            empties(*bad)


# ---------------------------------------------------------------------- the host module's way and the binding's
class Noted:
    """A library whose calls are noted with all their arguments."""

    def __init__(self):
        self.last = None

    def __getattr__(self, name):
        def call(*args):
            self.last = args
            return 0
        return call


class Like(Stand):
    """A stand-in for a tensor, contiguous where that is (strides of a single element say nothing)."""

    def __init__(self, t):
        super().__init__(t.dtype, tuple(t.shape), t.stride(), t.data_ptr())
        self.is_contiguous = t.is_contiguous


def as_stand(t):
    return Like(t) if isinstance(t, torch.Tensor) else t


def both(monkeypatch, name, fast, slow, args, results):
    """The arguments that reach the C ABI by either way (None: refused), results as their number."""
    from paper_1903_05133_gb300 import _lib
    host = _lib.host()
    host.pretend(True)
    try:
        made = getattr(host, fast)(*args)
    finally:
        noted = host.pretend(False)
    def plainly(call, outs):
        at = {t.data_ptr(): f"result {i}" for i, t in enumerate(outs) if t is not None and t.numel()}
        return [at.get(a, a) for a in call]
    first = None
    if made is not None:
        first = plainly(noted, made if isinstance(made, tuple) else (made,))
    library, stands = Noted(), []

    def empties(like, *specs):
        kinds = (F, BF, HF, I32, torch.uint8)
        out = tuple(Stand(kinds[q[0]], q[1:], address=(1 << 50) + i * (1 << 40)) for i, q in enumerate(specs))
        stands.extend(out)
        return out
    with monkeypatch.context() as m:
        m.setattr(ops._lib, "load", lambda: library)
        m.setattr(ops, "_empties", empties)
        m.setattr(ops, "_CURRENT", lambda: 0)
        m.setattr(ops, "_RAW_STREAM", lambda d: 0)
        try:
            slow(*[as_stand(a) for a in args])
            second = plainly(library.last, stands[:results])
        except (ValueError, AttributeError, TypeError):
            second = None
    return first, second, made is not None


def same(first, second):
    """Equal but for the workspace's address, and results without elements."""
    if len(first) != len(second):
        return False
    number = lambda a: 0 if a is None else getattr(a, "value", a)  # noqa: E731
    for a, b in zip(map(number, first), map(number, second)):
        far = isinstance(b, int) and b >= 1 << 50
        if a != b and not far and not (isinstance(a, str) or isinstance(b, str)):
            return False
    return True


def test_the_host_module_takes_what_the_binding_takes(lib, monkeypatch):
    """Random calls, most of them with something wrong: what the host module takes reaches the C ABI as the binding
    would send it, and what the binding refuses it does not take."""
    import random

    from paper_1903_05133_gb300 import _lib
    _lib.host()
    rng = random.Random(11)
    pick = lambda *v: rng.choice(v)  # noqa: E731
    wrong = lambda p=0.06: rng.random() < p  # noqa: E731

    def tensor(dtype, *shape):
        """Contiguous or with gaps, sometimes of another type, size, order or none at all."""
        if wrong(0.02):
            return None
        if wrong():
            dtype = pick(torch.float64, torch.int64, torch.int16, F, BF, I32)
        shape = [max(n + pick(-1, 1), 0) if wrong(0.03) else n for n in shape]
        t = torch.zeros(*shape, dtype=dtype)
        if len(shape) >= 2 and rng.random() < 0.25:
            wide = torch.zeros(*shape[:-1], shape[-1] + 5, dtype=dtype)
            t = wide[..., 2:2 + shape[-1]]
        if wrong(0.03) and t.dim() >= 2:
            t = t.transpose(-1, -2)
        if wrong(0.03) and t.dim() >= 1:
            t = t[..., ::2]
        if wrong(0.02):
            t = t.unsqueeze(0)
        if wrong(0.03) and t.dim() >= 2:
            t = t[:1].expand(*t.shape) if t.shape[0] else t
        return t
    taken = refused = 0
    for _ in range(6000):
        T, k, E, D, G = pick(0, 1, 2, 5, 40, 300), pick(1, 2, 3, 8), pick(1, 3, 8, 64), pick(1, 7, 16), pick(1, 4, 9)
        B, K, V = pick(0, 1, 3), pick(0, 1, 4), pick(1, 5, 30)
        kind, over = pick(F, BF, HF), pick(True, False)
        word = "all" if over else "chosen"
        out_dtype = pick(None, kind, F, HF, torch.float64)
        temperature = pick(1.0, 0.5, 1e27, 2.0 ** -126, 0.0, -1.0, 1e28, float("nan"))
        one, maybe = tensor, lambda *a: None if rng.random() < 0.4 else tensor(*a)  # noqa: E731
        ok = pick(None, one(torch.bool, V), one(torch.uint8, B, K + 1, V), torch.zeros(B, 1, V, dtype=torch.bool).expand(-1, K + 1, -1),
                  torch.zeros(V, dtype=torch.bool).expand(B, K + 1, V))
        name, fast, slow, args, results = pick(
            lambda: ("route", "route", lambda z, n, o, p: ops.route(z, n, over=word, learners=p),
                     (one(kind, T, E), pick(k, 0, 33, -1) if wrong() else k, over, maybe(I32, G + 1)), 6),
            lambda: ("route_backward", "route_backward", lambda dw, z, e, w, s, o: ops.route_backward(dw, z, e, w, lse=s, over=word),
                     (one(F, T, k), one(kind, T, E), one(I32, T, k), one(F, T, k), maybe(F, T), over), 1),
            lambda: ("dispatch", "dispatch", ops.dispatch, (one(kind, T, D), one(I32, T, k), one(I32, G + 1)), 1),
            lambda: ("combine", "combine", lambda y, p, w, d: ops._combine("y", y, p, w, None, d, None),
                     (one(kind, T * k, D), one(I32, T, k), maybe(F, T, k), out_dtype), 1),
            lambda: ("combine_backward", "combine_backward", ops.combine_backward,
                     (one(pick(kind, F), T, D), one(kind, T * k, D), one(I32, T, k), one(F, T, k), one(I32, G + 1)), 2),
            lambda: ("verify_drafts", "verify", lambda z, x, u, n, q, t, a: ops.verify_drafts(z, x, u, n, draft_probs=q, temperature=t, allowed=a),
                     (one(kind, B, K + 1, V), one(pick(I32, torch.int64), B, K), one(F, B, K), one(F, B, V),
                      maybe(pick(F, BF, HF), B, K, V), temperature, ok), 3))()
        first, second, went = both(monkeypatch, name, fast, slow, args, results)
        shown = [(tuple(a.shape), a.dtype, a.stride()) if isinstance(a, torch.Tensor) else a for a in args]
        if went:
            assert second is not None, (name, shown)
            assert same(first, second), (name, shown, first, second)
            taken += 1
        else:
            refused += second is None
    assert taken > 1500 and refused > 1500, (taken, refused)


def test_norm_by_the_host_module(lib):
    from paper_1903_05133_gb300 import _lib
    host = _lib.host()
    g = [torch.zeros(4, 3), torch.zeros(4, 2, dtype=BF)]
    assert host.norm(g, 1.0, None, False) is None            # not on a GPU
    host.pretend(True)
    try:
        norm, scale = host.norm(g, 2.5, 4, True)
        assert tuple(norm.shape) == tuple(scale.shape) == (4,) and norm.dtype == scale.dtype == F
        noted = host.pretend(True)
        assert noted[0] == 2 and noted[4:7] == (4, 2.5, 1) and noted[7] == norm.data_ptr() and noted[8] == scale.data_ptr()
        assert host.norm(g, None, None, False)[1] is None and host.pretend(True)[8] == 0
        # the workspace is as large as the library says, or larger
        import random
        rng, need = random.Random(3), ctypes.c_int64()
        for _ in range(300):
            P_, count, most = rng.choice((1, 1, 3, 16)), rng.randint(1, 40), rng.choice((3, 600, 5000, 100000))
            kinds = [rng.choice((F, BF, HF)) for _ in range(count)]
            some = [torch.empty(P_, rng.randint(0, most) // P_, dtype=d) for d in kinds]
            assert host.norm(some, 1.0, P_, False) is not None
            given = host.pretend(True)[10]
            sizes, types = (ctypes.c_int64 * count)(*[t.numel() for t in some]), (ctypes.c_int * count)(*[ops.TYPES[d] for d in kinds])
            assert lib.hier_avg_grad_norm_workspace(count, types, sizes, P_, ctypes.byref(need)) == 0
            assert need.value <= given <= 4 * need.value + 64 * count * P_
        for bad in (([], 1.0, None, False), (g, -1.0, None, False), (g, float("nan"), None, False), (g, float("inf"), None, False),
                    (g, 1, None, False), (g, 1.0, 3, False), (g, 1.0, 0, False), (g, 1.0, 2.0, False), (g + [torch.zeros(())], 1.0, 4, False),
                    (g + [None], 1.0, None, False), (g + [torch.zeros(4, dtype=torch.float64)], 1.0, None, False),
                    ([torch.zeros(4, 3).T], 1.0, None, False), (iter(g), 1.0, None, False), (g, 1.0, None)):
            assert host.norm(*bad) is None, bad
    finally:
        host.pretend(False)
