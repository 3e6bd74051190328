"""What the operators' binding refuses before it calls the library, on stand-ins for CUDA tensors: no
address is read here."""
import pytest
import torch

from paper_1903_05133_gb300 import operators as ops

BF, HF, F, I32, BOOL = torch.bfloat16, torch.float16, torch.float32, torch.int32, torch.bool


class Stand:
    """A CUDA tensor as far as its type, shape, strides and address go."""
    is_cuda = True

    def __init__(self, dtype, shape, strides=None, address=1 << 20, gpu=0):
        self.dtype, self.shape, self.address, self.gpu = dtype, torch.Size(shape), address, gpu
        if strides is None:
            strides = [1]
            for n in reversed(shape[1:]):
                strides.insert(0, strides[0] * n)
        self.strides = tuple(strides[:len(shape)])

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return Stand(self.dtype, self.shape).strides == self.strides or 0 in self.shape

    def element_size(self):
        return self.dtype.itemsize

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self.gpu


def test_masks_with_overlapping_rows_are_refused():
    T, V = 6, 100
    logits, targets = Stand(BF, (T, V)), Stand(I32, (T,))
    given = lambda *a, **k: ops._logits(logits, targets, Stand(BOOL, *a, **k), 1.0)[1:]  # noqa: E731
    for stride in (1, 50, V - 1):                           # a sliding window's 1
        with pytest.raises(ValueError, match="overlap"):
            given((T, V), (stride, 1))
    at = 1 << 20
    assert given((T, V)) == (at, V) and given((T, V), (V + 3, 1)) == (at, V + 3)
    assert given((V,)) == (at, 0) and given((T, V), (0, 1)) == (at, 0)
    one = Stand(BF, (1, V)), Stand(I32, (1,))               # the stride of one row says nothing
    assert ops._logits(*one, Stand(BOOL, (1, V), (1, 1)), 1.0)[1:] == (at, 0)


def test_adamw_eps_without_a_finite_reciprocal_is_refused(lib):
    import ctypes

    from test_operators_abi import EINVAL, create
    rc, h = create(lib)
    assert rc == 0
    g = (ctypes.c_void_p * 1)(4096)
    step = lambda eps: lib.hier_avg_adamw_step(h, g, 0, 0.1, 0.9, 0.99, eps, 1, None, 0, None)  # noqa: E731
    for eps in (2.0 ** -127, 1e-40, 1e-60, 0.0, float("nan")):
        assert step(eps) == EINVAL, eps
    assert step(2.0 ** -126) == step(1e-8) == -4            # HA_ESTATE: not bound
    lib.hier_avg_adamw_destroy(h)
    with pytest.raises(ValueError, match="eps"):
        ops.AdamW([Stand(F, (4,))], eps=1e-40)


def test_temperatures_without_a_finite_inverse_or_that_let_masked_classes_in_are_refused(lib):
    import ctypes

    from test_operators_abi import EINVAL, P
    fwd = lambda t, rows=0: lib.hier_avg_token_logprobs(P, 1, rows, 100, 100, P, 4, None, 0, t, 3, P, P, P, P, P, None)  # noqa: E731
    bwd = lambda t: lib.hier_avg_token_logprobs_backward(P, 1, 0, 100, 100, P, 4, None, 0, t, P, P, P, P, P, 100, None)  # noqa: E731
    logits, targets = Stand(BF, (3, 10)), Stand(I32, (3,))
    for t in (2.0 ** -127, 1e-45, 1.1e27, 3e38, float("inf"), float("nan"), -1.0, 0.0):
        t = ctypes.c_float(t).value
        assert fwd(t) == EINVAL and bwd(t) == EINVAL, t
        with pytest.raises(ValueError, match="temperature"):
            ops._logits(logits, targets, None, t)
    for t in (2.0 ** -126, 1.0, 9.9e26):
        assert fwd(t) == 0 and bwd(t) == 0, t
        ops._logits(logits, targets, None, t)


def test_weights_whose_groups_overlap_are_copied_first(lib):
    # a tensor map of them would have overlapping dimensions
    import ctypes
    G, N, K, T = 5, 24, 64, 40
    n = ctypes.c_int64(-1)

    def bytes_of(ld, gs, N=N, G=G):
        seen = set()
        for op, cols in ((ops.FORWARD, K), (ops.DX, N)):
            a = ctypes.c_void_p(1 << 20)
            assert lib.hier_avg_grouped_product_workspace(op, a, 64, a, ld, gs, G, T, K, N, ctypes.byref(n)) == 0
            seen.add(n.value - ops._copy_bytes(1 << 20, 1, T, cols, 64, 0))
        assert seen == {ops._copy_bytes(1 << 20, G, N, K, ld, gs)}
        return seen.pop()
    copy = -(-G * N * K * 2 // 256) * 256
    assert bytes_of(K, N * K) == 0 and bytes_of(K + 8, N * (K + 8)) == 0
    assert bytes_of(K, (N - 1) * K + K) == 0 and bytes_of(G * K, K) == 0        # rows of the groups in turn
    for ld, gs in ((K, 0), (K, 8), (K, K), (K, (N - 1) * K), (G * K - 8, K), (G * K, K - 8)):
        assert bytes_of(ld, gs) == copy, (ld, gs)
    assert bytes_of(K, K, N=1) == 0 and bytes_of(K, K - 8, N=1) > 0 and bytes_of(K, 8, G=1) == 0


class Calls:
    """A stand-in for the library that notes each call's name, the current GPU and the stream."""

    def __init__(self, gpus):
        self.gpus, self.made = gpus, []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, self.gpus[0], args[-1]))
            return 0
        return call


class Guard:
    def __init__(self, gpus, gpu):
        self.gpus, self.gpu = gpus, gpu

    def __enter__(self):
        self.before, self.gpus[0] = self.gpus[0], self.gpu

    def __exit__(self, *_):
        self.gpus[0] = self.before


class Stream:
    def __init__(self, gpu, handle):
        self.device_index, self.cuda_stream = gpu, handle


@pytest.fixture
def two_gpus(monkeypatch):
    """GPU 0 is current; the current stream of GPU d is 100 + d."""
    gpus = [0]
    calls = Calls(gpus)
    monkeypatch.setattr(ops._lib, "load", lambda: calls)
    monkeypatch.setattr(ops, "_CURRENT", lambda: gpus[0], raising=False)
    monkeypatch.setattr(ops, "_RAW_STREAM", lambda d: 100 + d)
    monkeypatch.setattr(ops, "_DEVICE", Stand.get_device, raising=False)
    monkeypatch.setattr(ops, "_ADDRESS", Stand.data_ptr)
    monkeypatch.setattr(ops, "_CONTIGUOUS", Stand.is_contiguous)
    monkeypatch.setattr(torch.cuda, "device", lambda d: Guard(gpus, d))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: Guard(gpus, s.device_index))
    return gpus, calls


def all_calls():
    """Each operator's arguments on GPU `gpu(name)`, aligned and with all its tensors given."""
    T, G, N, K, V = 6, 2, 16, 24, 40
    at = iter(range(1 << 20, 1 << 30, 1 << 20))

    def tensors(gpu):
        S = lambda name, dtype, shape: Stand(dtype, shape, address=next(at), gpu=gpu(name))  # noqa: E731
        off = lambda: S("offsets", I32, (G + 1,))  # noqa: E731
        opt = ops.AdamW.__new__(ops.AdamW)
        opt.h, opt._lib, opt.t, opt.bits, opt.beta1, opt.beta2, opt.eps = None, ops._lib.load(), 0, 32, 0.9, 0.99, 1e-8
        opt._kinds = {F: [(F, torch.Size((4,)))] * 2}
        opt._devices = [gpu("params")] * 2
        v = lambda name: S(name, F, (T,))  # noqa: E731
        return {
            "grouped_product": lambda **k: ops.grouped_product(
                S("x", BF, (T, K)), S("w", BF, (G, N, K)), off(), bias=S("bias", F, (G, N)), out=S("out", BF, (T, N)), **k),
            "grouped_product_dx": lambda **k: ops.grouped_product_dx(
                S("dy", BF, (T, N)), S("w", BF, (G, N, K)), off(), h=S("h", BF, (T, K)), out=S("out", BF, (T, K)), **k),
            "grouped_product_dw": lambda **k: ops.grouped_product_dw(
                S("dy", BF, (T, N)), S("x", BF, (T, K)), off(), out=S("out", BF, (G, N, K)), **k),
            "token_logprobs_backward": lambda **k: ops.token_logprobs_backward(
                S("logits", BF, (T, V)), S("targets", I32, (T,)), v("lse"), v("entropy"), v("dlogp"), v("dentropy"),
                allowed=S("allowed", BOOL, (T, V)), out=S("out", BF, (T, V)), **k),
            "adamw_step": lambda **k: opt.step([S("grads", F, (4,)), S("grads", F, (4,))], lr=0.1, grad_scale=S("grad_scale", F, (1,)), **k)}
    return tensors


def test_calls_run_on_their_tensors_gpu(two_gpus):
    gpus, calls = two_gpus
    for gpu in (0, 1):
        for name, call in all_calls()(lambda _: gpu).items():
            calls.made.clear()
            call()
            assert calls.made == [("hier_avg_" + name, gpu, 100 + gpu)] and gpus == [0], name
            calls.made.clear()
            call(stream=Stream(gpu, 7))
            assert calls.made == [("hier_avg_" + name, gpu, 7)] and gpus == [0], name
            calls.made.clear()
            with pytest.raises(ValueError, match="stream"):
                call(stream=Stream(1 - gpu, 7))
            assert not calls.made


def test_tensors_of_two_gpus_are_refused(two_gpus):
    gpus, calls = two_gpus
    seen = set()
    named = {"grouped_product": ("x", "w", "offsets", "bias", "out"), "grouped_product_dx": ("dy", "w", "offsets", "h", "out"),
             "grouped_product_dw": ("dy", "x", "offsets", "out"), "adamw_step": ("grads", "grad_scale", "params"),
             "token_logprobs_backward": ("logits", "targets", "lse", "entropy", "dlogp", "dentropy", "allowed", "out")}
    for name, tensors in named.items():
        for one in tensors:
            with pytest.raises(ValueError, match="GPU"):
                all_calls()(lambda n: int(n == one))[name]()
            seen.add((name, one))
    assert not calls.made and len(seen) == sum(map(len, named.values()))
    with pytest.raises(ValueError, match="GPU"):
        ops.token_logprobs(Stand(BF, (3, 8)), Stand(I32, (3,), gpu=1))


def test_results_that_share_memory_with_an_input_are_refused(two_gpus):
    gpus, calls = two_gpus
    T, G, N, K, at = 6, 2, 32, 32, 1 << 20
    far = iter(range(1 << 24, 1 << 30, 1 << 20))
    S = lambda dtype, shape, address=None, strides=None: Stand(  # noqa: E731
        dtype, shape, strides, next(far) if address is None else address)
    off = S(I32, (G + 1,))
    product = lambda out, x=None, w=None, o=off, b=None: ops.grouped_product(  # noqa: E731
        x or S(BF, (T, K)), w or S(BF, (G, N, K)), o, bias=b, out=out)
    x, w, b = S(BF, (T, K), at), S(BF, (G, N, K), at), S(F, (G, N), at)
    for kw in (dict(x=x), dict(w=w), dict(b=b), dict(o=S(I32, (G + 1,), at))):
        for place in (0, 2, -(T * N * 2) + 2):
            with pytest.raises(ValueError, match="share"):
                product(S(BF, (T, N), at + place), **kw)
    dy, h = S(BF, (T, N)), S(BF, (T, K), at)
    with pytest.raises(ValueError, match="share"):
        ops.grouped_product_dx(dy, S(BF, (G, N, K)), off, h=h, out=S(BF, (T, K), at + 2 * K))
    with pytest.raises(ValueError, match="share"):
        ops.grouped_product_dx(dy, S(BF, (G, N, K)), off, h=h, out=S(F, (T, K), at))
    with pytest.raises(ValueError, match="share"):
        ops.grouped_product_dx(S(BF, (T, N), at), S(BF, (G, N, K)), off, out=S(BF, (T, K), at))
    with pytest.raises(ValueError, match="share"):
        ops.grouped_product_dw(dy, S(BF, (T, K), at + 64), off, out=S(BF, (G, N, K), at))
    v = S(F, (T,))
    grad = lambda logits, out, lse=v: ops.token_logprobs_backward(logits, S(I32, (T,)), lse, None, v, out=out)  # noqa: E731
    for out, lse in ((S(BF, (T, N), at + 2 * N), v), (S(BF, (T, N), at, (2 * N, 1)), v), (S(BF, (T, N)), None)):
        with pytest.raises(ValueError, match="share"):
            grad(S(BF, (T, N), at), out, lse or S(F, (T,), out.address))
    assert not calls.made
    # what is side by side in one buffer, after one another, or the same where that is allowed
    side = lambda i, n=32, dtype=BF: S(dtype, (T, n), at + 64 * i, (96, 1))  # noqa: E731
    product(side(1), x=side(0))
    product(side(0), x=side(2))
    product(S(BF, (T, N), at + T * K * 2), x=x)
    ops.grouped_product_dx(dy, S(BF, (G, N, K)), off, h=h, out=S(BF, (T, K), at))
    ops.grouped_product_dw(dy, S(BF, (T, K), at, (96, 1)), off, out=S(BF, (G, N, K), at + 64, (N * 96, 96, 1)))
    grad(S(BF, (T, N), at), S(BF, (T, N), at))
    grad(side(0), side(1))
    grad(S(BF, (T, N), at), S(BF, (T, N), at + T * N * 2))
    with pytest.raises(ValueError, match="share"):          # a mask of one row for all
        ops.token_logprobs_backward(S(BF, (T, N)), S(I32, (T,)), v, None, v, allowed=Stand(BOOL, (T, N), (0, 1), at),
                                    out=S(BF, (T, N), at))
    assert len(calls.made) == 8
    with pytest.raises(ValueError, match="share"):
        product(side(1, 33), x=side(2))


def test_adamw_parameters_that_share_memory_are_refused(lib):
    at = 1 << 20
    p = lambda n, address: Stand(F, (n,), None, address)  # noqa: E731
    for params, copies in (([p(8, at), p(8, at)], None), ([p(8, at), p(4, at + 28)], None),
                           ([p(8, at), p(8, at + 64)], [None, Stand(BF, (8,), None, at + 16)]),
                           ([p(8, at), p(8, at + 64)], [Stand(BF, (8,), None, at + 128), Stand(BF, (8,), None, at + 140)])):
        with pytest.raises(ValueError, match="share"):
            ops.AdamW(params, copies=copies)


def test_adamw_plans_beyond_any_memory_are_refused_at_once(lib):
    from test_operators_abi import EINVAL, create
    for n in ((1 << 62,), (1 << 38,), (100, 1 << 37)):
        rc, h = create(lib, n=n, tensor=(0,) * len(n), decay=(0.0,) * len(n), offset=(0,) * len(n))
        assert rc == EINVAL and not h.value, n
