"""Operators for models with grouped weights: products by group with their gradients, log
probabilities of given classes with their gradient, and AdamW over many tensors.

Argument marshalling only, as in hier_avg.py: PyTorch provides the memory and the stream, the
computation runs in the library's CUDA kernels, and the functions are those of
include/hier_avg.h without the ``hier_avg_`` prefix.  Results are new tensors unless ``out``
is given.  A call on ``stream`` makes its results and workspace there.
"""
from __future__ import annotations

import ctypes
from contextlib import nullcontext
from typing import Dict, List, NamedTuple, Optional, Sequence

import torch

from . import _lib
from ._lib import c_int64, c_void_p, check

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
FORWARD, DX, DW = 0, 1, 2
BLOCK = 256                     # elements that share a scale of the 8-bit AdamW states
MAX_TOP = 32


def _on(stream):
    """The stream's handle and a context that allocates on it."""
    if stream is None:
        return torch.cuda.current_stream().cuda_stream, nullcontext()
    return stream.cuda_stream, torch.cuda.stream(stream)


def _need(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _rows_of(name: str, t: torch.Tensor, dtypes, rows: Optional[int] = None,
             cols: Optional[int] = None) -> None:
    """t is a CUDA matrix of one of the types whose rows have unit stride."""
    _need(t.is_cuda and t.dim() == 2 and t.dtype in dtypes,
          f"{name} must be a CUDA matrix of {' or '.join(str(d) for d in dtypes)}")
    _need(rows is None or t.shape[0] == rows, f"{name} must have {rows} rows")
    _need(cols is None or t.shape[1] == cols, f"{name} must have {cols} columns")
    _need(t.shape[1] >= 1 and (t.stride(1) == 1 or t.shape[1] == 1),
          f"{name} must have columns of unit stride")
    _need(t.shape[0] <= 1 or t.stride(0) >= t.shape[1], f"{name}'s rows must not overlap")


def _ld(t: torch.Tensor) -> int:
    """Elements between rows (the width where there is one row and the stride says nothing)."""
    return max(t.stride(-2), t.shape[-1]) if t.shape[-2] > 1 else t.shape[-1]


def _result(out, shape, dtype, device, name="out"):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _need(out.is_cuda and tuple(out.shape) == tuple(shape) and out.dtype == dtype and
          (out.stride(-1) == 1 or shape[-1] == 1), f"{name} must be {dtype} {list(shape)} with unit column stride")
    _need(all(out.stride(i) >= out.shape[i + 1] * max(out.stride(i + 1), 1)
              for i in range(out.dim() - 1) if out.shape[i] > 1), f"{name}'s rows must not overlap")
    return out


# ---------------------------------------------------------------------- grouped products
_HALF = (torch.bfloat16, torch.float16)


def _grouped(rows_t, w, offsets, name):
    _need(w.is_cuda and w.dim() == 3 and w.dtype == rows_t.dtype,
          f"w must be a CUDA tensor [groups, outer, inner] of {name}'s type")
    _need(min(w.shape) >= 1 and (w.stride(2) == 1 or w.shape[2] == 1), "w must have rows of unit stride")
    _need((w.shape[1] == 1 or w.stride(1) >= w.shape[2]) and w.stride(0) >= 0, "w's rows must not overlap")
    _offsets(offsets, w.shape[0])


def _offsets(offsets, groups):
    _need(offsets.is_cuda and offsets.dtype == torch.int32 and offsets.dim() == 1 and
          offsets.is_contiguous(), "offsets must be a contiguous CUDA int32 vector")
    _need(groups is None or offsets.shape[0] == groups + 1, "offsets must have one entry more than there are groups")
    _need(offsets.shape[0] >= 2, "offsets must name at least one group")


def _out_type(out_dtype, out, dtype):
    d = out_dtype if out_dtype is not None else (out.dtype if out is not None else dtype)
    _need(d in (dtype, torch.float32), f"the result is {dtype} or torch.float32")
    return d


def _aligned(t: torch.Tensor) -> bool:
    return t.data_ptr() % 16 == 0 and all(
        t.stride(i) % 8 == 0 and t.stride(i) > 0 for i in range(t.dim() - 1) if t.shape[i] > 1)


def _workspace(lib, op, a, b, groups, rows, inner, outer, device):
    n = c_int64()
    check(lib.hier_avg_grouped_product_workspace(
        op, a.data_ptr(), _ld(a), b.data_ptr(), _ld(b), b.stride(0) if b.dim() == 3 else 0, groups,
        rows, inner, outer, ctypes.byref(n)), "grouped_product_workspace")
    return (torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None), n.value


def grouped_product(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, relu: bool = False,
                    out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                    stream=None) -> torch.Tensor:
    """y[t] = act(w[g] x[t] + bias[g]) for the rows t in [offsets[g], offsets[g+1]) of group g.

    x [rows, inner] and w [groups, outer, inner] bf16 or fp16, with any strides between rows and
    groups; offsets [groups + 1] int32 on the device; bias [groups, outer] fp32.  The result is
    of x's type or fp32; rows of no group are zero."""
    lib = _lib.load()
    _rows_of("x", x, _HALF)
    _grouped(x, w, offsets, "x")
    G, N, K = w.shape
    _need(x.shape[1] == K, f"x must have {K} columns, as w")
    if bias is not None:
        _rows_of("bias", bias, (torch.float32,), G, N)
    d = _out_type(out_dtype, out, x.dtype)
    T = x.shape[0]
    s, where = _on(stream)
    with where:
        y = _result(out, (T, N), d, x.device)
        ws, n = (None, 0) if _aligned(x) and _aligned(w) else _workspace(lib, FORWARD, x, w, G, T, K, N, x.device)
    check(lib.hier_avg_grouped_product(
        x.data_ptr(), _ld(x), w.data_ptr(), _ld(w), w.stride(0), TYPES[x.dtype], offsets.data_ptr(), G,
        T, K, N, bias.data_ptr() if bias is not None else None, _ld(bias) if bias is not None else 0,
        int(relu), y.data_ptr(), _ld(y), TYPES[d], ws.data_ptr() if n else None, n, s), "grouped_product")
    return y


def grouped_product_dx(dy: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor,
                       h: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """dx[t] = w[g]^T dy[t] for the rows of group g; with h [rows, inner] (the activations that
    grouped_product read, after a ReLU) zero where h is not positive."""
    lib = _lib.load()
    _rows_of("dy", dy, _HALF)
    _grouped(dy, w, offsets, "dy")
    G, N, K = w.shape
    _need(dy.shape[1] == N, f"dy must have {N} columns, as w has rows")
    T = dy.shape[0]
    if h is not None:
        _rows_of("h", h, (dy.dtype,), T, K)
    d = _out_type(out_dtype, out, dy.dtype)
    s, where = _on(stream)
    with where:
        dx = _result(out, (T, K), d, dy.device)
        ws, n = (None, 0) if _aligned(dy) and _aligned(w) else _workspace(lib, DX, dy, w, G, T, K, N, dy.device)
    check(lib.hier_avg_grouped_product_dx(
        dy.data_ptr(), _ld(dy), w.data_ptr(), _ld(w), w.stride(0), TYPES[dy.dtype], offsets.data_ptr(), G,
        T, K, N, h.data_ptr() if h is not None else None, _ld(h) if h is not None else 0, dx.data_ptr(),
        _ld(dx), TYPES[d], ws.data_ptr() if n else None, n, s), "grouped_product_dx")
    return dx


def grouped_product_dw(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor,
                       bias_grad: bool = False, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, stream=None):
    """dw[g] = sum of dy[t] x[t]^T over group g's rows, [groups, outer, inner] in dy's type or fp32;
    with bias_grad the pair (dw, db), db[g] = sum of dy[t] in fp32.  Empty groups give zero."""
    lib = _lib.load()
    _rows_of("dy", dy, _HALF)
    _rows_of("x", x, (dy.dtype,), dy.shape[0])
    _offsets(offsets, None)
    T, N, K, G = dy.shape[0], dy.shape[1], x.shape[1], offsets.shape[0] - 1
    d = _out_type(out_dtype, out, dy.dtype)
    s, where = _on(stream)
    with where:
        dw = _result(out, (G, N, K), d, dy.device)
        db = torch.empty(G, N, dtype=torch.float32, device=dy.device) if bias_grad else None
        ws, n = (None, 0) if T == 0 or (_aligned(dy) and _aligned(x)) else _workspace(lib, DW, dy, x, G, T, K, N, dy.device)
    check(lib.hier_avg_grouped_product_dw(
        dy.data_ptr(), _ld(dy), x.data_ptr(), _ld(x), TYPES[dy.dtype], offsets.data_ptr(), G, T, K, N,
        dw.data_ptr(), _ld(dw), dw.stride(0), TYPES[d], db.data_ptr() if bias_grad else None, N,
        ws.data_ptr() if n else None, n, s), "grouped_product_dw")
    return (dw, db) if bias_grad else dw


# ---------------------------------------------------------------------- log probabilities
class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                        # [rows] of the targets
    entropy: torch.Tensor                     # [rows]
    lse: torch.Tensor                         # [rows] log of the sum of the exponentials
    top_logp: Optional[torch.Tensor]          # [rows, top], falling
    top_index: Optional[torch.Tensor]         # [rows, top] int32, -1 where there is none


def _logits(logits, targets, allowed, temperature):
    _rows_of("logits", logits, tuple(TYPES))
    T, V = logits.shape
    _need(targets.is_cuda and targets.dtype in (torch.int32, torch.int64) and
          tuple(targets.shape) == (T,) and targets.is_contiguous(),
          "targets must be a contiguous CUDA int32 or int64 vector, one entry a row")
    _need(0 < temperature < float("inf"), "temperature must be positive and finite")
    if allowed is None:
        return None, 0
    _need(allowed.is_cuda and allowed.dtype in (torch.bool, torch.uint8) and
          tuple(allowed.shape) in ((V,), (T, V)) and (allowed.stride(-1) == 1 or V == 1),
          "allowed must be a CUDA bool tensor [classes] or [rows, classes] with unit stride in rows")
    if allowed.dim() == 1 or (T > 1 and allowed.stride(0) == 0):
        return allowed.data_ptr(), 0
    return allowed.data_ptr(), _ld(allowed)


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, top: int = 0, temperature: float = 1.0,
                   allowed: Optional[torch.Tensor] = None, stream=None) -> TokenLogprobs:
    """Log probability of each row's target under softmax(logits / temperature), the row's entropy,
    its log-sum-exp, and the ``top`` likeliest classes (equal logits by index).

    logits [rows, classes] fp32, bf16 or fp16; targets int32 or int64, below 0 for no target (logp 0);
    allowed: a mask [classes] or [rows, classes], False where a class is left out."""
    lib = _lib.load()
    mask, mask_ld = _logits(logits, targets, allowed, temperature)
    _need(0 <= top <= MAX_TOP, f"top must be in [0, {MAX_TOP}]")
    T, V = logits.shape
    s, where = _on(stream)
    with where:
        r = torch.empty(3, T, dtype=torch.float32, device=logits.device)
        best = torch.empty(T, top, dtype=torch.float32, device=logits.device) if top else None
        index = torch.empty(T, top, dtype=torch.int32, device=logits.device) if top else None
    p = r.data_ptr()
    check(lib.hier_avg_token_logprobs(
        logits.data_ptr(), TYPES[logits.dtype], T, V, _ld(logits), targets.data_ptr(),
        targets.element_size(), mask, mask_ld, temperature, top, p, p + 4 * T, p + 8 * T,
        best.data_ptr() if top else None, index.data_ptr() if top else None, s), "token_logprobs")
    logp, entropy, lse = r.unbind(0)
    return TokenLogprobs(logp, entropy, lse, best, index)


def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                            entropy: Optional[torch.Tensor], dlogp: torch.Tensor,
                            dentropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                            allowed: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """The gradient of sum(dlogp * logp + dentropy * entropy) with respect to the logits, in their
    type, from token_logprobs's lse and entropy; ``out`` may be ``logits`` itself."""
    lib = _lib.load()
    mask, mask_ld = _logits(logits, targets, allowed, temperature)
    T, V = logits.shape
    _need(dentropy is None or entropy is not None, "the entropy's gradient needs the entropy")
    for name, v in (("lse", lse), ("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy)):
        _need(v is None or (v.is_cuda and v.dtype == torch.float32 and tuple(v.shape) == (T,) and
                            v.is_contiguous()), f"{name} must be a contiguous CUDA fp32 vector, one entry a row")
    s, where = _on(stream)
    with where:
        d = _result(out, (T, V), logits.dtype, logits.device)
    check(lib.hier_avg_token_logprobs_backward(
        logits.data_ptr(), TYPES[logits.dtype], T, V, _ld(logits), targets.data_ptr(),
        targets.element_size(), mask, mask_ld, temperature, lse.data_ptr(),
        entropy.data_ptr() if entropy is not None else None, dlogp.data_ptr(),
        dentropy.data_ptr() if dentropy is not None else None, d.data_ptr(), _ld(d), s),
        "token_logprobs_backward")
    return d


# ---------------------------------------------------------------------- AdamW
class AdamW:
    """AdamW over a list of fp32 tensors in one launch a step, with states in 32 or 8 bits.

    params: CUDA fp32 tensors, contiguous, or matrices with rows of unit stride (the layers of a
    learner-indexed parameter matrix, say).  copies: bf16 or fp16 tensors of the same shapes that
    each step writes too (None: none), as the products read them.  decay: one weight decay for
    all tensors, or one a tensor.

    State: ``m`` and ``v`` (fp32), or in 8 bits ``m`` and ``root`` (e4m3, the first moment and the square
    root of the second) with ``m_scale`` and ``root_scale`` for each block of 256 elements; the
    pieces (whole tensors, or rows of a strided one) follow one another from multiples of 256."""

    def __init__(self, params: Sequence[torch.Tensor], bits: int = 32, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, decay=0.0,
                 copies: Optional[Sequence[Optional[torch.Tensor]]] = None, stream=None):
        self.h = c_void_p()
        lib = self._lib = _lib.load()
        params = list(params)
        _need(len(params) >= 1, "params must not be empty")
        _need(bits in (8, 32), "bits must be 8 or 32")
        _need(0 <= beta1 < 1 and 0 <= beta2 < 1 and 0 < eps < float("inf"), "betas must be in [0, 1), eps positive")
        decays = [float(decay)] * len(params) if isinstance(decay, (int, float)) else [float(d) for d in decay]
        copies = [None] * len(params) if copies is None else list(copies)
        _need(len(decays) == len(params) and len(copies) == len(params), "decay and copies must be one a tensor")
        kinds = {c.dtype for c in copies if c is not None}
        _need(len(kinds) <= 1 and kinds <= set(_HALF), "copies must be all bf16 or all fp16")
        tensor: List[int] = []
        addr: List[int] = []
        copy: List[int] = []
        size: List[int] = []
        offset: List[int] = []
        weight: List[float] = []
        for i, (p, c) in enumerate(zip(params, copies)):
            _need(p.is_cuda and p.dtype == torch.float32, "params must be CUDA fp32 tensors")
            _need(c is None or (c.is_cuda and c.shape == p.shape), "a copy must have its tensor's shape")
            for a, o, b, n in _pieces(p, c):
                tensor.append(i)
                addr.append(a)
                offset.append(o)
                copy.append(b)
                size.append(n)
                weight.append(decays[i])
        n = len(tensor)
        arr = lambda kind, v: (kind * max(n, 1))(*v)  # noqa: E731
        check(lib.hier_avg_adamw_create(
            bits, len(params), n, arr(ctypes.c_int, tensor), arr(c_void_p, addr),
            arr(c_void_p, copy) if kinds else None, TYPES[kinds.pop()] if kinds else 0,
            arr(c_int64, size), arr(c_int64, offset), arr(ctypes.c_float, weight),
            ctypes.byref(self.h)), "adamw_create")
        elements, table = c_int64(), c_int64()
        check(lib.hier_avg_adamw_sizes(self.h, ctypes.byref(elements), ctypes.byref(table)), "adamw_sizes")
        self.params, self.copies, self.bits = params, copies, bits
        self.beta1, self.beta2, self.eps, self.t = beta1, beta2, eps, 0
        e, dev = elements.value, params[0].device
        s, where = _on(stream)
        with where:
            self._table = torch.empty(max(table.value, 16), dtype=torch.uint8, device=dev)
            self.m_scale = self.root_scale = self.v = self.root = None
            if bits == 32:
                self.m = torch.zeros(e, device=dev)
                self.v = torch.zeros(e, device=dev)
            else:
                self.m = torch.zeros(e, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
                self.root = torch.zeros(e, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
                self.m_scale = torch.zeros(e // BLOCK, device=dev)
                self.root_scale = torch.zeros(e // BLOCK, device=dev)
        second = self.v if bits == 32 else self.root
        check(lib.hier_avg_adamw_bind(
            self.h, self._table.data_ptr(), table.value, self.m.data_ptr(), second.data_ptr(),
            self.m_scale.data_ptr() if bits == 8 else None,
            self.root_scale.data_ptr() if bits == 8 else None, s), "adamw_bind")
        self._grads = (c_void_p * len(params))()

    def step(self, grads: Sequence[torch.Tensor], lr: float, grad_scale: Optional[torch.Tensor] = None,
             seed: Optional[int] = None, stream=None) -> None:
        """One step from contiguous gradients of the params' shapes, all fp32, bf16 or fp16, times
        grad_scale (one fp32 value on the device) where given.  seed: of the 8-bit states' rounding
        (the step's number when None); the same seed gives the same step."""
        _need(len(grads) == len(self.params), "one gradient a tensor")
        kind = grads[0].dtype
        _need(kind in TYPES, "gradients must be fp32, bf16 or fp16")
        a = self._grads
        for i, (g, p) in enumerate(zip(grads, self.params)):
            if not (g.is_cuda and g.dtype == kind and g.shape == p.shape and g.is_contiguous()):
                raise ValueError(f"gradient {i} must be a contiguous CUDA {kind} tensor {list(p.shape)}")
            a[i] = g.data_ptr()
        if grad_scale is not None:
            _need(grad_scale.is_cuda and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1,
                  "grad_scale must be one CUDA fp32 value")
        s = (torch.cuda.current_stream() if stream is None else stream).cuda_stream
        check(self._lib.hier_avg_adamw_step(
            self.h, a, TYPES[kind], lr, self.beta1, self.beta2, self.eps, self.t + 1,
            grad_scale.data_ptr() if grad_scale is not None else None,
            (self.t + 1 if seed is None else seed) & 0xFFFFFFFF, s), "adamw_step")
        self.t += 1

    def state_dict(self) -> Dict[str, object]:
        """The step count and the state arrays themselves (not copies)."""
        names = ("m", "v") if self.bits == 32 else ("m", "m_scale", "root", "root_scale")
        return {"t": self.t, **{k: getattr(self, k) for k in names}}

    def load_state_dict(self, state: Dict[str, object]) -> None:
        """Copies a state_dict of an optimizer over the same pieces."""
        own = self.state_dict()
        _need(set(state) == set(own), f"the state must have {sorted(own)}")
        for k, v in own.items():
            if k != "t":
                _need(state[k].shape == v.shape and state[k].dtype == v.dtype, f"{k} must be {v.dtype} {list(v.shape)}")
        for k, v in own.items():
            if k != "t":
                v.copy_(state[k])
        self.t = int(state["t"])

    def destroy(self) -> None:
        if self.h:
            self._lib.hier_avg_adamw_destroy(self.h)
            self.h = c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _pieces(p: torch.Tensor, c: Optional[torch.Tensor]):
    """(address, first element of the gradient, the copy's address, elements) of each contiguous run."""
    if p.is_contiguous() and (c is None or c.is_contiguous()):
        return [(p.data_ptr(), 0, c.data_ptr() if c is not None else 0, p.numel())]
    ok = lambda t: t.dim() >= 1 and (t.shape[0] <= 1 or t.stride(0) >= t[0].numel()) and t[0].is_contiguous()  # noqa: E731
    _need(ok(p) and (c is None or ok(c)), "params and copies must be contiguous but for their first dimension's stride")
    n = p[0].numel()
    return [(p.data_ptr() + 4 * r * p.stride(0), r * n,
             c.data_ptr() + 2 * r * c.stride(0) if c is not None else 0, n) for r in range(p.shape[0])]


def operator_check(stream=None) -> None:
    """Synchronise the stream; raise if a bounded wait inside a grouped product ran out."""
    s = (torch.cuda.current_stream() if stream is None else stream).cuda_stream
    check(_lib.load().hier_avg_operator_check(s), "operator_check")
