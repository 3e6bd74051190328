"""Operators for models with grouped weights: products by group with their gradients, log
probabilities of given classes with their gradient, and AdamW over many tensors.

Argument marshalling only, as in hier_avg.py: PyTorch provides the memory and the stream, the
computation runs in the library's CUDA kernels, and the functions are those of
include/hier_avg.h without the ``hier_avg_`` prefix.  Results are new tensors unless ``out``
is given, and outside autograd: a result has no history even where an input requires gradients, whose
calls are grouped_product_dx, grouped_product_dw and token_logprobs_backward.  All tensors of a
call are on one GPU, where it runs whichever is current.  A call on ``stream`` makes its results and
workspace there; its inputs are the caller's to keep until it is done.
"""
from __future__ import annotations

import ctypes
from array import array
from contextlib import nullcontext
from operator import attrgetter
from typing import Dict, List, NamedTuple, Optional, Sequence

import torch

from . import _lib
from ._lib import c_int64, c_void_p, check

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
FORWARD, DX, DW = 0, 1, 2
_KIND = attrgetter("dtype", "shape")
_ADDRESS, _CONTIGUOUS, _DEVICE = torch.Tensor.data_ptr, torch.Tensor.is_contiguous, torch.Tensor.get_device
BLOCK = 256                     # elements that share a scale of the 8-bit AdamW states
MAX_TOP = 32


_NOWHERE = nullcontext()
_RAW_STREAM = torch._C._cuda_getCurrentRawStream    # current_stream() makes an object: 5 us
_CURRENT = torch._C._cuda_getDevice


def _on(stream, t, *others):
    """The stream's handle (the current one of t's GPU), and a context in which that GPU is current and
    allocations are the stream's.  The other tensors (or None) must be on the same GPU."""
    d = t.get_device()
    for o in others:
        if o is not None and o.get_device() != d:
            raise ValueError("all tensors of a call must be on one GPU")
    if stream is None:
        return _RAW_STREAM(d), _NOWHERE if d == _CURRENT() else torch.cuda.device(d)
    if stream.device_index != d:
        raise ValueError("stream must be of the tensors' GPU")
    return stream.cuda_stream, torch.cuda.stream(stream)


def _need(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _rows_of(name: str, t: torch.Tensor, dtypes, rows: Optional[int] = None,
             cols: Optional[int] = None) -> int:
    """Elements between the rows of t, a CUDA matrix of one of the types whose rows have unit
    stride (the width where there is one row and the stride says nothing)."""
    if not (t.is_cuda and t.dim() == 2 and t.dtype in dtypes):
        raise ValueError(f"{name} must be a CUDA matrix of {' or '.join(str(d) for d in dtypes)}")
    (r, c), (ld, unit) = t.shape, t.stride()
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name} must be [{r if rows is None else rows}, {c if cols is None else cols}]")
    if c < 1 or (unit != 1 and c != 1):
        raise ValueError(f"{name} must have columns of unit stride")
    if r <= 1:
        return c
    if ld < c:
        raise ValueError(f"{name}'s rows must not overlap")
    return ld


def _ld(t: torch.Tensor) -> int:
    return max(t.stride(-2), t.shape[-1]) if t.shape[-2] > 1 else t.shape[-1]


def _given(out, shape, dtype):
    if not (out.is_cuda and tuple(out.shape) == shape and out.dtype == dtype and
            (out.stride(-1) == 1 or shape[-1] == 1)):
        raise ValueError(f"out must be {dtype} {list(shape)} with unit column stride")
    _need(all(out.stride(i) >= out.shape[i + 1] * max(out.stride(i + 1), 1)
              for i in range(out.dim() - 1) if out.shape[i] > 1), "out's rows must not overlap")
    return out


def _end(t, at):
    last = 1
    for n, s in zip(t.shape, t.stride()):
        last += (n - 1) * s
    return at + last * t.element_size()


def _pitch(t):
    """Bytes of a row and from row to row (None: there is one row, 0: they differ)."""
    es = t.element_size()
    rows = [s for n, s in zip(t.shape[:-1], t.stride()) if n > 1 and s > 0]
    if not rows:
        return es * t.shape[-1], None
    return es * t.shape[-1], 0 if any(s % rows[-1] for s in rows) else es * rows[-1]


def _apart(out, *inputs, same=None):
    """Refuses an out that shares memory with an input, unless it is `same` itself (which then is read
    before it is written, element by element)."""
    if out is None or not out.numel():
        return
    p = out.data_ptr()
    end = _end(out, p)
    for t in inputs:
        if t is None:
            continue
        q = t.data_ptr()
        if q >= end or _end(t, q) <= p or not t.numel():
            continue
        (width, step), (t_width, t_step) = _pitch(out), _pitch(t)
        if t is same and p == q and t.shape == out.shape and t.dtype == out.dtype and step == t_step:
            continue
        # columns of one buffer side by side
        step = step if t_step is None else t_step if step is None else step if step == t_step else 0
        _need(bool(step) and width <= (q - p) % step <= step - t_width, "out must not share memory with an input")


# ---------------------------------------------------------------------- grouped products
_HALF = (torch.bfloat16, torch.float16)


def _grouped(w, offsets, dtype, name):
    """Groups, outer, inner, the row and the group stride of w."""
    if not (w.is_cuda and w.dim() == 3 and w.dtype == dtype):
        raise ValueError(f"w must be a CUDA tensor [groups, outer, inner] of {name}'s type")
    (G, N, K), (gs, ld, unit) = w.shape, w.stride()
    if min(G, N, K) < 1 or (unit != 1 and K != 1):
        raise ValueError("w must have rows of unit stride")
    if N == 1:
        ld = K
    _need(ld >= K, "w's rows must not overlap")
    _offsets(offsets, G)
    return G, N, K, ld, gs


def _offsets(offsets, groups):
    if not (offsets.is_cuda and offsets.dtype == torch.int32 and offsets.dim() == 1 and
            offsets.is_contiguous()):
        raise ValueError("offsets must be a contiguous CUDA int32 vector")
    n = offsets.shape[0]
    _need(n >= 2 and (groups is None or n == groups + 1), "offsets must have one entry more than there are groups")
    return n - 1


def _out_type(out_dtype, out, dtype):
    d = out_dtype if out_dtype is not None else (out.dtype if out is not None else dtype)
    if d is not dtype and d is not torch.float32:
        raise ValueError(f"the result is {dtype} or torch.float32")
    return d


def _copy_bytes(address: int, groups: int, rows: int, cols: int, ld: int, gs: int) -> int:
    """What the copy of an operand takes, 0 where the kernels can read it in place: as
    hier_avg_grouped_product_workspace counts it, without the call (3 us of a small product's 20)."""
    if not (address & 15 or (ld | cols) & 7 or groups > 1 and (gs & 7 or gs < (rows - 1) * ld + cols and not (
            gs >= cols and ld >= (groups - 1) * gs + cols))):
        return 0
    return groups * rows * ((cols + 7) & ~7) * 2 + 255 & ~255


def _workspace(lib, op, a, a_ld, b, b_ld, b_gs, groups, rows, inner, outer):
    """Device memory for operands that have to be copied first and for sums in parts (None where
    there are none)."""
    if rows == 0:
        return None, None, 0
    if op == DW and rows >= 1024 * groups:                  # long groups may be summed in parts
        n = c_int64()
        check(lib.hier_avg_grouped_product_workspace(
            op, a.data_ptr(), a_ld, b.data_ptr(), b_ld, b_gs, groups, rows, inner, outer,
            ctypes.byref(n)), "grouped_product_workspace")
        n = n.value
    else:
        n = _copy_bytes(a.data_ptr(), 1, rows, inner if op == FORWARD else outer, a_ld, 0) + (
            _copy_bytes(b.data_ptr(), 1, rows, inner, b_ld, 0) if op == DW else
            _copy_bytes(b.data_ptr(), groups, outer, inner, b_ld, b_gs))
    if n == 0:
        return None, None, 0
    ws = torch.empty(n, dtype=torch.uint8, device=a.device)
    return ws, ws.data_ptr(), n


def grouped_product(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor,
                    bias: Optional[torch.Tensor] = None, relu: bool = False,
                    out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                    stream=None) -> torch.Tensor:
    """y[t] = act(w[g] x[t] + bias[g]) for the rows t in [offsets[g], offsets[g+1]) of group g.

    x [rows, inner] and w [groups, outer, inner] bf16 or fp16, with any strides between rows and
    groups; offsets [groups + 1] int32 on the device; bias [groups, outer] fp32.  The result is
    of x's type or fp32; rows of no group are zero."""
    lib = _lib.load()
    ld = _rows_of("x", x, _HALF)
    kind = x.dtype
    G, N, K, w_ld, gs = _grouped(w, offsets, kind, "x")
    T = x.shape[0]
    if x.shape[1] != K:
        raise ValueError(f"x must have {K} columns, as w")
    bias_ld = 0 if bias is None else _rows_of("bias", bias, (torch.float32,), G, N)
    d = _out_type(out_dtype, out, kind)
    _apart(out, x, w, offsets, bias)
    s, where = _on(stream, x, w, offsets, bias, out)
    with where:
        y = torch.empty((T, N), dtype=d, device=x.device) if out is None else _given(out, (T, N), d)
        ws, p, n = _workspace(lib, FORWARD, x, ld, w, w_ld, gs, G, T, K, N)
        check(lib.hier_avg_grouped_product(
            x.data_ptr(), ld, w.data_ptr(), w_ld, gs, TYPES[kind], offsets.data_ptr(), G, T, K, N,
            None if bias is None else bias.data_ptr(), bias_ld, relu, y.data_ptr(),
            N if out is None else _ld(y), TYPES[d], p, n, s), "grouped_product")
    return y


def grouped_product_dx(dy: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor,
                       h: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """dx[t] = w[g]^T dy[t] for the rows of group g; with h [rows, inner] (the activations that
    grouped_product read, after a ReLU) zero where h is not positive; ``out`` may be ``h`` itself."""
    lib = _lib.load()
    ld = _rows_of("dy", dy, _HALF)
    kind = dy.dtype
    G, N, K, w_ld, gs = _grouped(w, offsets, kind, "dy")
    T = dy.shape[0]
    if dy.shape[1] != N:
        raise ValueError(f"dy must have {N} columns, as w has rows")
    h_ld = 0 if h is None else _rows_of("h", h, (kind,), T, K)
    d = _out_type(out_dtype, out, kind)
    _apart(out, dy, w, offsets, h, same=h)
    s, where = _on(stream, dy, w, offsets, h, out)
    with where:
        dx = torch.empty((T, K), dtype=d, device=dy.device) if out is None else _given(out, (T, K), d)
        ws, p, n = _workspace(lib, DX, dy, ld, w, w_ld, gs, G, T, K, N)
        check(lib.hier_avg_grouped_product_dx(
            dy.data_ptr(), ld, w.data_ptr(), w_ld, gs, TYPES[kind], offsets.data_ptr(), G, T, K, N,
            None if h is None else h.data_ptr(), h_ld, dx.data_ptr(), K if out is None else _ld(dx),
            TYPES[d], p, n, s), "grouped_product_dx")
    return dx


def grouped_product_dw(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor,
                       bias_grad: bool = False, out: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, stream=None):
    """dw[g] = sum of dy[t] x[t]^T over group g's rows, [groups, outer, inner] in dy's type or fp32;
    with bias_grad the pair (dw, db), db[g] = sum of dy[t] in fp32.  Empty groups give zero."""
    lib = _lib.load()
    ld = _rows_of("dy", dy, _HALF)
    kind, (T, N) = dy.dtype, dy.shape
    x_ld = _rows_of("x", x, (kind,), T)
    G, K = _offsets(offsets, None), x.shape[1]
    d = _out_type(out_dtype, out, kind)
    _apart(out, dy, x, offsets)
    s, where = _on(stream, dy, x, offsets, out)
    with where:
        dw = torch.empty((G, N, K), dtype=d, device=dy.device) if out is None else _given(out, (G, N, K), d)
        db = torch.empty((G, N), dtype=torch.float32, device=dy.device) if bias_grad else None
        ws, p, n = _workspace(lib, DW, dy, ld, x, x_ld, 0, G, T, K, N)
        dw_ld, dw_gs = (K, N * K) if out is None else (_ld(dw), dw.stride(0))
        check(lib.hier_avg_grouped_product_dw(
            dy.data_ptr(), ld, x.data_ptr(), x_ld, TYPES[kind], offsets.data_ptr(), G, T, K, N,
            dw.data_ptr(), dw_ld, dw_gs, TYPES[d], db.data_ptr() if bias_grad else None, N, p, n, s),
            "grouped_product_dw")
    return (dw, db) if bias_grad else dw


# ---------------------------------------------------------------------- log probabilities
class TokenLogprobs(NamedTuple):
    logp: torch.Tensor                        # [rows] of the targets
    entropy: torch.Tensor                     # [rows]
    lse: torch.Tensor                         # [rows] log of the sum of the exponentials
    top_logp: Optional[torch.Tensor]          # [rows, top], falling
    top_index: Optional[torch.Tensor]         # [rows, top] int32, -1 where there is none


def _logits(logits, targets, allowed, temperature):
    """The logits' row stride, the mask's address and its row stride."""
    ld = _rows_of("logits", logits, TYPES)
    T, V = logits.shape
    if not (targets.is_cuda and targets.dtype in (torch.int32, torch.int64) and
            targets.dim() == 1 and targets.shape[0] == T and targets.is_contiguous()):
        raise ValueError("targets must be a contiguous CUDA int32 or int64 vector, one entry a row")
    _need(2.0 ** -126 <= temperature <= 1e27, "temperature must be in [2^-126, 1e27]")
    if allowed is None:
        return ld, None, 0
    if not (allowed.is_cuda and allowed.dtype in (torch.bool, torch.uint8) and
            tuple(allowed.shape) in ((V,), (T, V)) and (allowed.stride(-1) == 1 or V == 1)):
        raise ValueError("allowed must be a CUDA bool tensor [classes] or [rows, classes] with unit stride in rows")
    if allowed.dim() == 1 or T <= 1 or allowed.stride(0) == 0:
        return ld, allowed.data_ptr(), 0
    _need(allowed.stride(0) >= V, "allowed's rows must not overlap")
    return ld, allowed.data_ptr(), allowed.stride(0)


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, top: int = 0, temperature: float = 1.0,
                   allowed: Optional[torch.Tensor] = None, stream=None) -> TokenLogprobs:
    """Log probability of each row's target under softmax(logits / temperature), the row's entropy,
    its log-sum-exp, and the ``top`` likeliest classes (equal logits by index).

    logits [rows, classes] fp32, bf16 or fp16; targets int32 or int64, below 0 for no target (logp 0);
    allowed: a mask [classes] or [rows, classes], False where a class is left out."""
    lib = _lib.load()
    ld, mask, mask_ld = _logits(logits, targets, allowed, temperature)
    if not 0 <= top <= MAX_TOP:
        raise ValueError(f"top must be in [0, {MAX_TOP}]")
    T, V = logits.shape
    s, where = _on(stream, logits, targets, allowed)
    best = index = b = i = None
    with where:
        dev = logits.device
        # three tensors and not three rows of one: a view costs more than an allocation
        logp = torch.empty(T, dtype=torch.float32, device=dev)
        entropy = torch.empty(T, dtype=torch.float32, device=dev)
        lse = torch.empty(T, dtype=torch.float32, device=dev)
        if top:
            best = torch.empty((T, top), dtype=torch.float32, device=dev)
            index = torch.empty((T, top), dtype=torch.int32, device=dev)
            b, i = best.data_ptr(), index.data_ptr()
        check(lib.hier_avg_token_logprobs(
            logits.data_ptr(), TYPES[logits.dtype], T, V, ld, targets.data_ptr(), targets.element_size(), mask, mask_ld,
            temperature, top, logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), b, i, s), "token_logprobs")
    return TokenLogprobs(logp, entropy, lse, best, index)


def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                            entropy: Optional[torch.Tensor], dlogp: torch.Tensor,
                            dentropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                            allowed: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    """The gradient of sum(dlogp * logp + dentropy * entropy) with respect to the logits, in their
    type, from token_logprobs's lse and entropy; ``out`` may be ``logits`` itself."""
    lib = _lib.load()
    ld, mask, mask_ld = _logits(logits, targets, allowed, temperature)
    T, V = logits.shape
    _need(dentropy is None or entropy is not None, "the entropy's gradient needs the entropy")
    for name, v in (("lse", lse), ("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy)):
        if v is not None and not (v.is_cuda and v.dtype == torch.float32 and v.dim() == 1 and
                                  v.shape[0] == T and v.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous CUDA fp32 vector, one entry a row")
    _apart(out, logits, targets, allowed, lse, entropy, dlogp, dentropy, same=logits)
    s, where = _on(stream, logits, targets, allowed, lse, entropy, dlogp, dentropy, out)
    with where:
        d = torch.empty((T, V), dtype=logits.dtype, device=logits.device) if out is None else \
            _given(out, (T, V), logits.dtype)
        check(lib.hier_avg_token_logprobs_backward(
            logits.data_ptr(), TYPES[logits.dtype], T, V, ld, targets.data_ptr(),
            targets.element_size(), mask, mask_ld, temperature, lse.data_ptr(),
            None if entropy is None else entropy.data_ptr(), dlogp.data_ptr(),
            None if dentropy is None else dentropy.data_ptr(), d.data_ptr(),
            V if out is None else _ld(d), s), "token_logprobs_backward")
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
        _need(0 <= beta1 < 1 and 0 <= beta2 < 1 and 2.0 ** -126 <= eps < float("inf"),
              "betas must be in [0, 1), eps at least 2^-126 and finite")
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
        # each element is changed by one thread
        spans = sorted([(a, a + 4 * n) for a, n in zip(addr, size) if n] + [(b, b + 2 * n) for b, n in zip(copy, size) if b and n])
        _need(all(a[1] <= b[0] for a, b in zip(spans, spans[1:])), "params and copies must not share memory")
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
        s, where = _on(stream, *params, *copies)
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
        self._kinds = {d: [(d, p.shape) for p in params] for d in TYPES}
        self._devices = [params[0].get_device()] * len(params)

    def step(self, grads: Sequence[torch.Tensor], lr: float, grad_scale: Optional[torch.Tensor] = None,
             seed: Optional[int] = None, stream=None) -> None:
        """One step from contiguous gradients of the params' shapes, all fp32, bf16 or fp16, times
        grad_scale (one fp32 value on the device) where given.  seed: of the 8-bit states' rounding
        (the step's number when None); the same seed gives the same step."""
        # each check runs over all tensors at once: a call over hundreds of them is host work
        kind = grads[0].dtype if grads else None
        if not (kind in TYPES and list(map(_KIND, grads)) == self._kinds[kind] and
                list(map(_DEVICE, grads)) == self._devices and all(map(_CONTIGUOUS, grads))):
            raise ValueError("grads must be one contiguous tensor on the params' GPU for each of them, of "
                             "its shape, all of them fp32, bf16 or fp16")
        a = array("Q", map(_ADDRESS, grads))
        if grad_scale is not None:
            _need(grad_scale.is_cuda and grad_scale.dtype == torch.float32 and grad_scale.numel() == 1,
                  "grad_scale must be one CUDA fp32 value")
        s, where = _on(stream, grads[0], grad_scale)
        with where:
            check(self._lib.hier_avg_adamw_step(
                self.h, a.buffer_info()[0], TYPES[kind], lr, self.beta1, self.beta2, self.eps, self.t + 1,
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
    """Synchronise the stream; raise if a bounded wait inside a grouped product ran out.  The GPU keeps
    one note for all streams: what another one's work has left there is reported, and cleared, too."""
    stream = torch.cuda.current_stream() if stream is None else stream
    with torch.cuda.device(stream.device):
        check(_lib.load().hier_avg_operator_check(stream.cuda_stream), "operator_check")
