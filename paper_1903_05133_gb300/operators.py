"""Operators for models with grouped weights: products by group with their gradients, the router that
makes the groups and the rows' way there and back with theirs, log probabilities of given classes with
their gradient, drafted tokens verified, the norm of all gradients, and AdamW over many tensors.

Argument marshalling only, as in hier_avg.py: PyTorch provides the memory and the stream, the
computation runs in the library's CUDA kernels, and the functions are those of
include/hier_avg.h without the ``hier_avg_`` prefix.  Results are new tensors unless ``out``
is given, and outside autograd: a result has no history even where an input requires gradients, whose
calls are grouped_product_dx, grouped_product_dw and the functions that end in _backward.  Autograd does not see
what is written into an ``out``, by clip_gradients or by AdamW.step either (no version counter moves): such a tensor must
not be saved for a backward pass that is still to come.  The usual calls of the
routing, row, norm and draft operators go through the host module at once; what it does not take (another stream, an
``out``, anything to refuse) goes through the checks here.  Results of such a call that are below 4 MB together are parts of
one allocation, which lives as long as any of them (and which torch.save writes as a whole: clone what is to be kept alone).
All tensors of a
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
_F32, _I32, _U8 = 0, 3, 4       # of results made together
_SMALL_WORK = 8192              # bytes of a workspace that may share the results' memory
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


def _empties(like, *specs):
    """New tensors on like's GPU of (type, size, ...) each, in one call (1.6 us each otherwise)."""
    return _lib.host().empties(like, *specs)


def _with_workspace(like, n, *specs):
    """_empties, and n bytes that the results do not hold where they are many (as the host module makes them)."""
    if n <= _SMALL_WORK:
        return _empties(like, *specs, (_U8, n))
    return *_empties(like, *specs), _empties(like, (_U8, n))[0]


def _empty(like, rows, cols, dtype):
    return _empties(like, (TYPES[dtype], rows, cols))[0]


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


# ---------------------------------------------------------------------- routing
class Routing(NamedTuple):
    experts: torch.Tensor                     # [rows, k] int32, -1 where there is none
    weights: torch.Tensor                     # [rows, k]
    lse: torch.Tensor                         # [rows] log of the sum of the exponentials
    offsets: torch.Tensor                     # [groups + 1] int32, as the grouped products read them
    place: torch.Tensor                       # [rows, k] int32, each entry's among the sorted, -1: none
    source: torch.Tensor                      # [rows * k] int32, the entry at each place, -1 behind the last


class Sorted(NamedTuple):
    offsets: torch.Tensor
    place: torch.Tensor
    source: torch.Tensor


MAX_CHOSEN, MAX_GROUPS = 32, 1024
_ONE_ROWS, _ONE_ENTRIES = 32, 1024


def _vector(name, t, dtype, shape):
    if not (t.is_cuda and t.dtype == dtype and tuple(t.shape) == shape and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous CUDA {dtype} tensor {list(shape)}")


def _sort_bytes(lib, rows, k, groups):
    if rows <= _ONE_ROWS and rows * k <= _ONE_ENTRIES:      # one CTA sorts them: none, as the library says
        return 0
    if rows * k <= 1 << 27:                                 # at most 153 chunks' counts, without the call
        return 4 * 154 * groups
    n = c_int64()
    check(lib.hier_avg_sort_workspace(rows, k, groups, ctypes.byref(n)), "sort_workspace")
    return n.value


def _over(over):
    _need(over in ("chosen", "all"), "over must be 'chosen' or 'all'")
    return over == "all"


def route(logits: torch.Tensor, k: int, over: str = "chosen", learners: Optional[torch.Tensor] = None,
          stream=None) -> Routing:
    """The k experts of largest logits for each row (equal logits by index), their weights, and the entries
    sorted by expert for dispatch, the grouped products and combine.

    logits [rows, experts] fp32, bf16 or fp16, at or below -1e30 where masked; the weights are softmax over the
    ``chosen`` or over ``all`` experts.  learners [learners + 1] int32 on the device, rising: the rows of
    each learner, which has experts of its own (group = learner * experts + expert)."""
    every = _over(over)
    if stream is None:
        r = _lib.host().route(logits, k, every, learners)
        if r is not None:
            return Routing(*r)
    lib = _lib.load()
    ld = _rows_of("logits", logits, TYPES)
    T, E = logits.shape
    _need(1 <= k <= min(E, MAX_CHOSEN), f"k must be in [1, {min(E, MAX_CHOSEN)}]")
    P = 0 if learners is None else _offsets(learners, None)
    G = E * max(P, 1)
    _need(G <= MAX_GROUPS, f"there must be at most {MAX_GROUPS} groups")
    s, where = _on(stream, logits, learners)
    with where:
        n = _sort_bytes(lib, T, k, G)
        experts, weights, lse, offsets, place, source, ws = _with_workspace(
            logits, n, (_I32, T, k), (_F32, T, k), (_F32, T), (_I32, G + 1), (_I32, T, k), (_I32, T * k))
        check(lib.hier_avg_route(
            logits.data_ptr(), TYPES[logits.dtype], T, E, ld, k, every, None if learners is None else learners.data_ptr(), P,
            experts.data_ptr(), weights.data_ptr(), lse.data_ptr(), offsets.data_ptr(), place.data_ptr(),
            source.data_ptr(), ws.data_ptr(), n, s), "route")
    return Routing(experts, weights, lse, offsets, place, source)


def route_backward(dweights: torch.Tensor, logits: torch.Tensor, experts: torch.Tensor, weights: torch.Tensor,
                   lse: Optional[torch.Tensor] = None, over: str = "chosen", out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """The gradient of sum(dweights * weights) with respect to the logits, in their type, from route's experts and
    weights (and lse for over="all"); ``out`` may be ``logits`` itself."""
    every = _over(over)
    if stream is None and out is None:
        r = _lib.host().route_backward(dweights, logits, experts, weights, lse, every)
        if r is not None:
            return r
    lib = _lib.load()
    ld = _rows_of("logits", logits, TYPES)
    T, E = logits.shape
    _need(experts.dim() == 2, "experts must be [rows, k]")
    k = experts.shape[1]
    _need(1 <= k <= min(E, MAX_CHOSEN), f"k must be in [1, {min(E, MAX_CHOSEN)}]")
    _vector("experts", experts, torch.int32, (T, k))
    _vector("weights", weights, torch.float32, (T, k))
    _vector("dweights", dweights, torch.float32, (T, k))
    _need(lse is not None or not every, "over='all' needs lse")
    if lse is not None:
        _vector("lse", lse, torch.float32, (T,))
    _apart(out, dweights, logits, experts, weights, lse, same=logits)
    s, where = _on(stream, logits, dweights, experts, weights, lse, out)
    with where:
        d = _empty(logits, T, E, logits.dtype) if out is None else _given(out, (T, E), logits.dtype)
        check(lib.hier_avg_route_backward(
            dweights.data_ptr(), logits.data_ptr(), TYPES[logits.dtype], T, E, ld, k, every, experts.data_ptr(),
            weights.data_ptr(), None if lse is None else lse.data_ptr(), d.data_ptr(), E if out is None else _ld(d), s),
            "route_backward")
    return d


def sort_by_group(group: torch.Tensor, groups: int, stream=None) -> Sorted:
    """The sort of route for given groups [rows, k] int32 (a router of the caller's own, or route's experts
    after some were dropped); below 0 or from ``groups`` on: none."""
    lib = _lib.load()
    _need(group.dim() == 2, "group must be [rows, k]")
    T, k = group.shape
    _vector("group", group, torch.int32, (T, k))
    _need(1 <= k <= MAX_CHOSEN, f"k must be in [1, {MAX_CHOSEN}]")
    _need(1 <= groups <= MAX_GROUPS, f"groups must be in [1, {MAX_GROUPS}]")
    s, where = _on(stream, group)
    with where:
        n = _sort_bytes(lib, T, k, groups)
        offsets, place, source, ws = _with_workspace(group, n, (_I32, groups + 1), (_I32, T, k), (_I32, T * k))
        check(lib.hier_avg_sort_by_group(group.data_ptr(), T, k, groups, offsets.data_ptr(), place.data_ptr(),
                                         source.data_ptr(), ws.data_ptr(), n, s), "sort_by_group")
    return Sorted(offsets, place, source)


# ---------------------------------------------------------------------- rows to their groups and back
def _places(place, entries=None):
    if not (place.is_cuda and place.dtype == torch.int32 and place.dim() == 2 and place.is_contiguous()):
        raise ValueError("place must be a contiguous CUDA int32 matrix [rows, k]")
    T, k = place.shape
    _need(k >= 1, "place must have columns")
    _need(entries is None or entries == T * k, "the sorted rows must be as many as place has entries")
    return T, k


def dispatch(x: torch.Tensor, place: torch.Tensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
    """xs[place[t, j]] = x[t], [rows * k, width]; the rows behind the last group, offsets[-1], are zero.

    x [rows, width] fp32, bf16 or fp16; place [rows, k] and offsets as of route or sort_by_group.  To drop an entry,
    sort again with its group below 0: a place that is only overwritten leaves a row of its group unwritten."""
    if stream is None and out is None:
        r = _lib.host().dispatch(x, place, offsets)
        if r is not None:
            return r
    lib = _lib.load()
    T, k = _places(place)
    ld = _rows_of("x", x, TYPES, T)
    G, D = _offsets(offsets, None), x.shape[1]
    _apart(out, x, place, offsets)
    s, where = _on(stream, x, place, offsets, out)
    with where:
        xs = _empty(x, T * k, D, x.dtype) if out is None else _given(out, (T * k, D), x.dtype)
        check(lib.hier_avg_dispatch(x.data_ptr(), TYPES[x.dtype], T, D, ld, place.data_ptr(), k, offsets.data_ptr(), G,
                                    xs.data_ptr(), D if out is None else _ld(xs), s), "dispatch")
    return xs


def _combine(name, y, place, weights, out, out_dtype, stream):
    if stream is None and out is None:
        r = _lib.host().combine(y, place, weights, out_dtype)
        if r is not None:
            return r
    lib = _lib.load()
    T, k = _places(place)
    ld = _rows_of(name, y, TYPES, T * k)
    D = y.shape[1]
    if weights is not None:
        _vector("weights", weights, torch.float32, (T, k))
    d = _out_type(out_dtype, out, y.dtype)
    _apart(out, y, place, weights)
    s, where = _on(stream, y, place, weights, out)
    with where:
        o = _empty(y, T, D, d) if out is None else _given(out, (T, D), d)
        check(lib.hier_avg_combine(y.data_ptr(), TYPES[y.dtype], T, D, ld, place.data_ptr(), k,
                                   None if weights is None else weights.data_ptr(), o.data_ptr(),
                                   D if out is None else _ld(o), TYPES[d], s), "combine")
    return o


def dispatch_backward(dxs: torch.Tensor, place: torch.Tensor, out: Optional[torch.Tensor] = None,
                      out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """dx[t] = sum over j of dxs[place[t, j]], in dxs's type or fp32."""
    return _combine("dxs", dxs, place, None, out, out_dtype, stream)


def combine(y: torch.Tensor, place: torch.Tensor, weights: torch.Tensor, out: Optional[torch.Tensor] = None,
            out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """out[t] = sum over j of weights[t, j] y[place[t, j]], in y's type or fp32.

    y [rows * k, width] fp32, bf16 or fp16, the sorted rows' results; place and weights [rows, k] as of route.  An entry
    without a place adds its weight times 0: a token whose logits held NaN has NaN weights, and is NaN here."""
    _need(weights is not None, "weights must be given")
    return _combine("y", y, place, weights, out, out_dtype, stream)


def combine_backward(dout: torch.Tensor, y: torch.Tensor, place: torch.Tensor, weights: torch.Tensor, offsets: torch.Tensor,
                     out: Optional[torch.Tensor] = None, stream=None):
    """(dy, dweights): dy[place[t, j]] = weights[t, j] dout[t] in y's type, zero behind the last group (``out`` is for
    dy), and dweights[t, j] = <dout[t], y[place[t, j]]>.  dout is of y's type or fp32."""
    if stream is None and out is None:
        r = _lib.host().combine_backward(dout, y, place, weights, offsets)
        if r is not None:
            return r
    lib = _lib.load()
    T, k = _places(place)
    ld = _rows_of("y", y, TYPES, T * k)
    D, kind = y.shape[1], y.dtype
    dout_ld = _rows_of("dout", dout, (kind, torch.float32), T, D)
    _vector("weights", weights, torch.float32, (T, k))
    G = _offsets(offsets, None)
    _apart(out, dout, y, place, weights, offsets)
    s, where = _on(stream, y, dout, place, weights, offsets, out)
    with where:
        if out is None:
            dy, dw = _empties(y, (TYPES[kind], T * k, D), (_F32, T, k))
        else:
            dy, dw = _given(out, (T * k, D), kind), _empty(y, T, k, torch.float32)
        check(lib.hier_avg_combine_backward(
            dout.data_ptr(), TYPES[dout.dtype], dout_ld, y.data_ptr(), TYPES[kind], T, D, ld, place.data_ptr(), k,
            weights.data_ptr(), offsets.data_ptr(), G, dy.data_ptr(), D if out is None else _ld(dy), dw.data_ptr(), s),
            "combine_backward")
    return dy, dw


# ---------------------------------------------------------------------- drafted tokens
class VerifiedDrafts(NamedTuple):
    tokens: torch.Tensor                      # [sequences, drafts + 1] int32: the accepted, the next, then -1
    accepted: torch.Tensor                    # [sequences] int32
    logp: torch.Tensor                        # [sequences, drafts + 1] of the tokens, 0 where there is none


def _three(name, t, dtypes, shape):
    """The strides of the first two dimensions of a CUDA tensor of unit stride in the last."""
    if not (t.is_cuda and t.dtype in dtypes and tuple(t.shape) == shape and (t.stride(-1) == 1 or shape[-1] == 1)):
        raise ValueError(f"{name} must be a CUDA tensor {list(shape)} of {' or '.join(str(d) for d in dtypes)} with unit stride "
                         "in its last dimension")
    return t.stride()[:-1]


def verify_drafts(logits: torch.Tensor, drafts: torch.Tensor, uniform: torch.Tensor, noise: torch.Tensor,
                  draft_probs: Optional[torch.Tensor] = None, temperature: float = 1.0,
                  allowed: Optional[torch.Tensor] = None, stream=None) -> VerifiedDrafts:
    """Which drafted tokens the target accepts, and the token that follows them.

    logits [sequences, K + 1, classes] fp32, bf16 or fp16 of the target, after the drafts before each row; drafts
    [sequences, K] int32 or int64, below 0 where there is none; draft_probs [sequences, K, classes] that they were drawn
    from (None: they are certain).  Draft i is accepted while uniform[i] * draft_probs[i, draft] < p[i, draft], p =
    softmax(logits / temperature) over the allowed classes; the next token is the first argmax of r / noise, r = p
    less draft_probs where positive after a rejection, else p.  uniform [sequences, K] in [0, 1), noise [sequences,
    classes] positive, exponential for a draw from r, both fp32.  K may be 0: one token is then drawn from p.
    allowed: a mask [classes] or [sequences, K + 1, classes], which may be expanded."""
    if stream is None:
        r = _lib.host().verify(logits, drafts, uniform, noise, draft_probs, temperature, allowed)
        if r is not None:
            return VerifiedDrafts(*r)
    lib = _lib.load()
    _need(logits.dim() == 3 and logits.shape[1] >= 1 and logits.shape[2] >= 1, "logits must be [sequences, drafts + 1, classes]")
    B, R, V = logits.shape
    K = R - 1
    z = _three("logits", logits, tuple(TYPES), (B, R, V))
    if not (drafts.is_cuda and drafts.dtype in (torch.int32, torch.int64) and tuple(drafts.shape) == (B, K) and
            drafts.is_contiguous()):
        raise ValueError(f"drafts must be a contiguous CUDA int32 or int64 tensor {[B, K]}")
    _vector("uniform", uniform, torch.float32, (B, K))
    noise_ld, = _three("noise", noise, (torch.float32,), (B, V))
    q = (0, 0) if draft_probs is None else _three("draft_probs", draft_probs, tuple(TYPES), (B, K, V))
    _need(2.0 ** -126 <= temperature <= 1e27, "temperature must be in [2^-126, 1e27]")
    ok = (0, 0)
    if allowed is not None and allowed.dim() == 1:
        _three("allowed", allowed, (torch.bool, torch.uint8), (V,))
    elif allowed is not None:
        ok = _three("allowed", allowed, (torch.bool, torch.uint8), (B, R, V))
    s, where = _on(stream, logits, drafts, uniform, noise, draft_probs, allowed)
    with where:
        n = B * (272 * R + 2052)                            # as hier_avg_verify_workspace says
        tokens, accepted, logp, ws = _with_workspace(logits, n, (_I32, B, R), (_I32, B), (_F32, B, R))
        check(lib.hier_avg_verify_drafts(
            logits.data_ptr(), TYPES[logits.dtype], B, K, V, *z, drafts.data_ptr(), drafts.element_size(), uniform.data_ptr(),
            noise.data_ptr(), noise_ld, None if draft_probs is None else draft_probs.data_ptr(),
            0 if draft_probs is None else TYPES[draft_probs.dtype], *q, None if allowed is None else allowed.data_ptr(), *ok,
            temperature, tokens.data_ptr(), accepted.data_ptr(), logp.data_ptr(), ws.data_ptr(), n, s), "verify_drafts")
    return VerifiedDrafts(tokens, accepted, logp)


# ---------------------------------------------------------------------- the norm of all gradients
class GradNorm(NamedTuple):
    norm: torch.Tensor                        # [1], or [learners]
    scale: Optional[torch.Tensor]             # max_norm / norm where that is below 1, else 1; as AdamW.step takes it


def _norm(grads, max_norm, learners, clip, stream):
    if stream is None:
        r = _lib.host().norm(grads, max_norm if max_norm is None else float(max_norm), learners, clip)
        if r is not None:
            return GradNorm(*r)
    lib = _lib.load()
    n = len(grads)
    _need(n >= 1, "grads must not be empty")
    address, types, sizes, d = _lib.host().facts(grads)
    _need(d != -2, "all tensors of a call must be on one GPU")
    if d < 0:
        raise ValueError("grads must be contiguous CUDA tensors of fp32, bf16 or fp16")
    P = 1
    if learners is not None:
        P = learners
        _need(P >= 1 and all(g.dim() >= 1 and g.shape[0] == P for g in grads), "the gradients' first dimension must be the learners'")
    _need(max_norm is None or 0 <= max_norm < float("inf"), "max_norm must be finite and not negative")
    b = c_int64()
    check(lib.hier_avg_grad_norm_workspace(n, types, sizes, P, ctypes.byref(b)), "grad_norm_workspace")
    s, where = _on(stream, grads[0])
    with where:
        norm, scale, ws = _with_workspace(grads[0], b.value, (_F32, P), (_F32, P))
        if max_norm is None:
            scale = None
        status = lib.hier_avg_grad_norm(n, address, types, sizes, P, 0.0 if max_norm is None else max_norm, clip,
                                        norm.data_ptr(), None if scale is None else scale.data_ptr(), ws.data_ptr(), b.value, s)
        _need(not (clip and status == -1), "gradients that are clipped must not share memory")
        check(status, "clip_gradients" if clip else "grad_norm")
    return GradNorm(norm, scale)


def grad_norm(grads: Sequence[torch.Tensor], max_norm: Optional[float] = None, learners: Optional[int] = None,
              stream=None) -> GradNorm:
    """The norm of all gradients together and, with max_norm, the factor that clips them to it, on the device.

    grads: contiguous fp32, bf16 or fp16 tensors, of types of their own; learners: their first dimension is the learner's,
    and each has a norm and a factor.  A norm that is NaN has factor 1, an infinite one 0."""
    return _norm(grads, max_norm, learners, False, stream)


def clip_gradients(grads: Sequence[torch.Tensor], max_norm: float, learners: Optional[int] = None, stream=None) -> GradNorm:
    """grad_norm, and the gradients multiplied by their factor in place (where it is not 1), unseen by
    autograd.  They must not share memory.
    AdamW.step(grads, lr, grad_scale=grad_norm(grads, max_norm).scale) does the same without this pass."""
    _need(max_norm is not None, "max_norm must be given")
    return _norm(grads, max_norm, learners, True, stream)


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
