"""Experts in training and in four bits: ctypes binding of include/ocean_experts.h.

Beside the routing and the grouped products of `routed` stand the losses that keep a router's experts evenly used, with the gradient of the
logits, and matrices in microscaled four bits: made from a matrix, read back, and multiplied with ragged groups of rows.  As there, every step runs in
the HIP library, on the current stream or the one given; outputs and workspaces are torch tensors of that stream, nothing synchronises, calls can be
captured into a graph, an `out` may not overlap what is read, and there is no CPU fallback.  The calls are no part of torch's autograd.

A training step's router, for logits [T, E] (dloss: float32 [2], the losses' factors):

    r = routed.route(logits, k)
    b = route_balance(logits, r)                                    # b.loss [2], b.counts [E], b.prob [E]
    ...                                                             # experts, combine_backward -> dval
    dlogits = route_balance_backward(b, r, logits, dloss, dval=dval)   # of the weights and of the losses, in one pass

Experts whose matrices w1 [E, F, D] are held in four bits, and the gradient of their rows:

    w = mx4_quantize(w1)
    h = grouped_matmul_mx4(x, w, r.expert_ptr, rows=r.token)
    h = grouped_matmul_mx4(mx4_quantize(x), w, r.expert_ptr, rows=r.token, dtype=x.dtype)   # rows in four bits as well
    dx = grouped_matmul_mx4(dh, w, r.expert_ptr, transposed=True)
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

from . import binding as _b
from . import routed as _r
from .binding import OceanError  # noqa: F401
from .routed import _at, _code, _groups, _matrix, _output, _ptr, _vector, ocean_groups, ocean_routing

BLOCK = 32   # numbers that share a scale


class ocean_balance(C.Structure):
    _fields_ = [("loss", C.c_void_p), ("counts", C.c_void_p), ("prob", C.c_void_p), ("rows", C.c_void_p)]


class ocean_mx4(C.Structure):
    _fields_ = [("count", C.c_int64), ("rows", C.c_int64), ("inner", C.c_int64), ("codes", C.c_void_p), ("ld_codes", C.c_int64), ("stride_codes", C.c_int64),
                ("scales", C.c_void_p), ("ld_scales", C.c_int64), ("stride_scales", C.c_int64)]


_lib = None


def load():
    """The HIP library with the argument types of ocean_experts.h set."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _r.load()
    P, vp, i64, i32, size = C.POINTER, C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
    lib.ocean_route_balance_workspace.argtypes = [i64, i64]
    lib.ocean_route_balance_workspace.restype = size
    lib.ocean_route_balance.argtypes = [P(ocean_routing), vp, i32, i64, P(ocean_balance), vp, size, vp]
    lib.ocean_route_balance_backward.argtypes = [P(ocean_balance), P(ocean_routing), vp, i32, i64, vp, vp, i32, vp, i64, vp]
    lib.ocean_mx4_quantize.argtypes = [vp, i32, i64, i64, P(ocean_mx4), vp]
    lib.ocean_mx4_dequantize.argtypes = [P(ocean_mx4), i32, vp, i64, i64, vp]
    lib.ocean_grouped_matmul_mx4.argtypes = [P(ocean_groups), i32, vp, i64, P(ocean_mx4), i32, vp, i64, vp]
    lib.ocean_grouped_matmul_mx4_mx4.argtypes = [P(ocean_groups), P(ocean_mx4), P(ocean_mx4), i32, vp, i64, vp]
    for name in ("ocean_route_balance", "ocean_route_balance_backward", "ocean_mx4_quantize", "ocean_mx4_dequantize", "ocean_grouped_matmul_mx4",
                 "ocean_grouped_matmul_mx4_mx4"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


# ---------------------------------------------------------------- balance
@dataclass(frozen=True)
class Balance:
    """How a router uses its experts: loss (float32 [2]: balance, logits' size), counts (int64 [experts]: entries of each), prob (float32 [experts]: mean
    probabilities), rows (int64 [1]: rows that have a logit which is not masked)."""
    loss: "object"
    counts: "object"
    prob: "object"
    rows: "object"


def route_balance(logits, routing, *, stream=None) -> Balance:
    """The losses of a routing made from logits [tokens, experts].  Over the rows with a logit that is not masked (NaN, -inf and the type's lowest value
    are): loss[0] = experts * sum of counts[e] / entries * prob[e], with prob[e] the mean of softmax(row)[e], and loss[1] = the mean of
    logsumexp(row)^2."""
    import torch
    lib = load()
    ld = _matrix(logits, "logits", routing.tokens, routing.experts)
    code = _code(logits.dtype)
    lists = routing._lists(logits.device)
    s, here = _at(logits.device, stream, logits, *lists)
    with here:
        E, dev = routing.experts, logits.device
        counts, rows = torch.empty(E, dtype=torch.int64, device=dev), torch.empty(1, dtype=torch.int64, device=dev)
        loss, prob = torch.empty(2, dtype=torch.float32, device=dev), torch.empty(E, dtype=torch.float32, device=dev)
        nbytes = lib.ocean_route_balance_workspace(routing.tokens, E)
        space = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        c = ocean_balance(loss.data_ptr(), counts.data_ptr(), prob.data_ptr(), rows.data_ptr())
        _b._check(lib.ocean_route_balance(C.byref(routing._struct()), _ptr(logits), code, ld, C.byref(c), space.data_ptr(), nbytes, s))
    return Balance(loss, counts, prob, rows)


def route_balance_backward(balance: Balance, routing, logits, dloss, *, dval=None, normalize: bool = True, out=None, stream=None):
    """Gradient of the logits from that of the losses, dloss (float32 [2]).  counts are constants; balance's counts and rows are used (a program
    on several devices puts the sums there), its loss and prob are not.  dval: float32 [tokens*k], the gradient of routing.val; then what
    routed.route_backward(routing, dval, logits, normalize=normalize) gives is added before the rounding.  Masked logits get 0."""
    import torch
    lib = load()
    ld = _matrix(logits, "logits", routing.tokens, routing.experts)
    code, dev = _code(logits.dtype), logits.device
    lists = routing._lists(dev)
    _vector(dloss, "dloss", torch.float32, 2, dev)
    _vector(balance.counts, "counts", torch.int64, routing.experts, dev)
    _vector(balance.rows, "rows", torch.int64, 1, dev)
    if dval is not None:
        if routing.val is None:
            raise ValueError("the routing has no weights")
        _vector(dval, "dval", torch.float32, routing.tokens * routing.k, dev)
    s, here = _at(dev, stream, logits, dloss, dval, out, balance.counts, balance.rows, *lists)
    with here:
        out = _output(out, logits.shape, logits)
        ldo = _matrix(out, "out", like=logits)
        c = ocean_balance(None, balance.counts.data_ptr(), None, balance.rows.data_ptr())
        _b._check(lib.ocean_route_balance_backward(C.byref(c), C.byref(routing._struct()), _ptr(logits), code, ld, dloss.data_ptr(), _ptr(dval),
                                                   int(normalize), _ptr(out), ldo, s))
    return out


# ---------------------------------------------------------------- four bits
def _blocks(inner: int) -> int:
    return (inner + BLOCK - 1) // BLOCK


def _apart(t, name, step):
    """(row stride, stride from one matrix to the next) in bytes of codes or scales; multiples of `step`, as the base is."""
    t = t if t.dim() == 3 else t.unsqueeze(0)
    n, rows, width = t.shape
    up = (width + step - 1) // step * step
    if t.numel() == 0:
        return up, rows * up
    ld, stride = t.stride(1) if rows > 1 else up, t.stride(0) if n > 1 else 0
    if width > 1 and t.stride(2) != 1:
        raise ValueError(f"{name}: the bytes of a row must be adjacent")
    if ld < width or (n > 1 and stride < 0):
        raise ValueError(f"{name}: rows overlap")
    if t.data_ptr() % step or ld % step or stride % step:
        raise ValueError(f"{name}: rows must begin at multiples of {step} bytes (Mx4.laid_out copies them so)")
    return max(ld, up), stride


@dataclass(frozen=True)
class Mx4:
    """A matrix [rows, inner] or matrices [count, rows, inner] in microscaled four bits (e2m1 codes with an e8m0 scale for every 32 numbers of a row).  codes:
    uint8 [.., rows, 16 * blocks], two numbers a byte, the earlier one in the low half, rows at multiples of 16 bytes; scales: uint8 [.., rows, blocks up to
    a multiple of 16] (those behind the blocks do not count), rows at multiples of 16 bytes; a number is its code's value times 2^(scale - 127), 255 makes a
    block of NaN.  blocks = (inner + 31) // 32, and codes behind `inner` do not count; shape is ((count,) rows, inner).  Slices of the matrices or of rows are made from slices of both arrays."""
    codes: "object"
    scales: "object"
    inner: int

    def __post_init__(self):
        import torch
        c, s, blocks = self.codes, self.scales, _blocks(self.inner)
        if c.dtype != torch.uint8 or s.dtype != torch.uint8 or c.dim() not in (2, 3) or s.dim() != c.dim() or c.shape[:-1] != s.shape[:-1]:
            raise ValueError(f"codes and scales must be uint8 [(count,) rows, bytes] of the same rows, not {c.dtype} {tuple(c.shape)} and {s.dtype} {tuple(s.shape)}")
        if self.inner < 0 or c.shape[-1] != 16 * blocks or s.shape[-1] < blocks or s.shape[-1] % 16:
            raise ValueError(f"rows of {self.inner} have {16 * blocks} bytes of codes and {blocks} scales up to a multiple of 16, not {c.shape[-1]} and {s.shape[-1]}")
        if c.device != s.device:
            raise ValueError(f"codes are on {c.device}, scales on {s.device}")
        ldc, sc = _apart(c, "codes", 16)
        lds, ss = _apart(s, "scales", 16)
        count, rows = (1, c.shape[0]) if c.dim() == 2 else c.shape[:2]
        self.__dict__.update(shape=(*c.shape[:-1], self.inner), _struct=ocean_mx4(count, rows, self.inner, _ptr(c), ldc, sc, _ptr(s), lds, ss))

    @classmethod
    def _made(cls, shape, device):
        """One with new arrays."""
        import torch
        *many, inner = shape
        blocks = _blocks(inner)
        width, up = 16 * blocks, (blocks + 15) // 16 * 16
        codes, scales = torch.empty((*many, width), dtype=torch.uint8, device=device), torch.empty((*many, up), dtype=torch.uint8, device=device)
        count, rows = many if len(many) == 2 else (1, many[0])
        q = object.__new__(cls)
        q.__dict__.update(codes=codes, scales=scales, inner=inner, shape=(*many, inner),
                          _struct=ocean_mx4(count, rows, inner, _ptr(codes), width, rows * width, _ptr(scales), up, rows * up))
        return q

    def __reduce__(self):
        """Copies and pickles are made of the fields: the struct holds pointers to this one's arrays."""
        return Mx4, (self.codes, self.scales, self.inner)

    @classmethod
    def laid_out(cls, codes, scales, inner: int) -> "Mx4":
        """Of codes [.., rows, 16 * blocks] and scales [.., rows, blocks] with any strides and alignment: copied where their rows do not lie as wanted."""
        import torch
        blocks = _blocks(inner)
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() not in (2, 3) or codes.shape[:-1] != scales.shape[:-1] or \
                codes.shape[-1] != 16 * blocks or scales.shape[-1] != blocks:
            raise ValueError(f"rows of {inner} have {16 * blocks} bytes of codes and {blocks} scales (uint8), not {tuple(codes.shape)} and {tuple(scales.shape)}")
        if blocks % 16:
            scales = torch.nn.functional.pad(scales, (0, 16 - blocks % 16))
        try:
            return cls(codes, scales, inner)
        except ValueError:
            copied = [torch.empty(t.shape, dtype=torch.uint8, device=t.device) for t in (codes, scales)]
            for to, t in zip(copied, (codes, scales)):
                to.copy_(t)
            return cls(*copied, inner)


def _cube(t, name, like=None):
    """(row stride, stride from one matrix to the next) of a matrix or matrices."""
    if t.dim() == 2:
        return _matrix(t, name, like=like), 0
    return _r._matrices(t, name, like=like)


def mx4_quantize(x, *, out: Mx4 = None, stream=None) -> Mx4:
    """x [rows, inner] or [count, rows, inner] in microscaled four bits: a block's scale is 2^(floor(log2 of its largest magnitude) - 2), numbers go to the nearest,
    ties to the even code, beyond 6 units to 6; a block with an infinite number or NaN becomes NaN."""
    import torch
    lib = load()
    if x.dim() not in (2, 3):
        raise ValueError(f"x must be [rows, inner] or [count, rows, inner], not {tuple(x.shape)}")
    code = _code(x.dtype)
    ld, stride = _cube(x, "x")
    held = () if out is None else (out.codes, out.scales)
    s, here = _at(x.device, stream, x, *held)
    with here:
        if out is None:
            out = Mx4._made(x.shape, x.device)
        elif tuple(out.shape) != tuple(x.shape) or out.codes.device != x.device:
            raise ValueError(f"out must be {tuple(x.shape)} on {x.device}, not {tuple(out.shape)} on {out.codes.device}")
        _b._check(lib.ocean_mx4_quantize(_ptr(x), code, ld, stride, C.byref(out._struct), s))
    return out


def mx4_dequantize(q: Mx4, dtype=None, *, out=None, stream=None):
    """The numbers of q in dtype (that of out; torch.bfloat16), rounded where it does not hold them."""
    import torch
    lib = load()
    dev = q.codes.device
    dtype = dtype or (out.dtype if out is not None else torch.bfloat16)
    code = _code(dtype)
    s, here = _at(dev, stream, q.codes, q.scales, out)
    with here:
        if out is None:
            out = torch.empty(q.shape, dtype=dtype, device=dev)
        elif tuple(out.shape) != q.shape or out.dtype != dtype or out.device != dev:
            raise ValueError(f"out must be {q.shape} {dtype} on {dev}, not {tuple(out.shape)} {out.dtype} on {out.device}")
        ld, stride = _cube(out, "out")
        _b._check(lib.ocean_mx4_dequantize(C.byref(q._struct), code, _ptr(out), ld, stride, s))
    return out


def grouped_matmul_mx4(x, w: Mx4, expert_ptr, *, rows=None, transposed: bool = False, dtype=None, out=None, stream=None):
    """As routed.grouped_matmul with matrices in four bits: y[s] = x[rows[s]] @ w[e].T for the slots s of expert e, or (transposed) x[rows[s]] @ w[e], which
    is the gradient of the rows.  w: Mx4 [experts, outer, inner].  x: a matrix [n, inner] ([n, outer] transposed) of float32, bfloat16 or float16, whose type the result
    has, or an Mx4 [n, inner] (not transposed), with the result's dtype (torch.bfloat16, or that of out).  Row numbers outside x stand for zeros; slots of no expert give zeros."""
    import torch
    lib = load()
    if len(w.shape) != 3:
        raise ValueError(f"w must be [experts, outer, inner], not {w.shape}")
    count, outer, inner = w.shape
    if transposed:
        outer, inner = inner, outer
    four = isinstance(x, Mx4)
    first = x.codes if four else x
    dev = first.device
    if four:
        if transposed or len(x.shape) != 2:
            raise ValueError("rows in four bits must be [n, inner], and are not multiplied with transposed matrices")
        dtype = dtype or (out.dtype if out is not None else torch.bfloat16)
    else:
        ldx = _matrix(x, "x")
        if dtype not in (None, x.dtype):
            raise ValueError(f"the result has the rows' type {x.dtype}, not {dtype}")
        dtype = x.dtype
    code = _code(dtype)
    g = _groups(first, expert_ptr, rows)
    if count != g.experts or inner != x.shape[1] or w.codes.device != dev:
        raise ValueError(f"w is {w.shape}{' (transposed)' if transposed else ''} on {w.codes.device}: not {g.experts} matrices for rows of {x.shape[1]} on {dev}")
    held = (x.codes, x.scales) if four else (x,)
    s, here = _at(dev, stream, *held, w.codes, w.scales, expert_ptr, rows, out)
    with here:
        if out is None:
            out = torch.empty((g.rows, outer), dtype=dtype, device=dev)
        elif tuple(out.shape) != (g.rows, outer) or out.dtype != dtype or out.device != dev:
            raise ValueError(f"out must be {(g.rows, outer)} {dtype} on {dev}, not {tuple(out.shape)} {out.dtype} on {out.device}")
        ldo = _matrix(out, "out")
        if four:
            _b._check(lib.ocean_grouped_matmul_mx4_mx4(C.byref(g), C.byref(x._struct), C.byref(w._struct), code, _ptr(out), ldo, s))
        else:
            _b._check(lib.ocean_grouped_matmul_mx4(C.byref(g), code, _ptr(x), ldx, C.byref(w._struct), int(transposed), _ptr(out), ldo, s))
    return out
