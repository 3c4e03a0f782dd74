"""Products in which every row chooses its matrix: ctypes binding of include/ocean_routed.h.

A routing matrix (tokens x experts, k entries a row) is made from logits, applied to the rows that the experts gave, and
differentiated; the ragged groups of rows that it forms are multiplied with their experts' weights; and rows that each name a
low-rank adapter are projected with it.  Every step runs in the HIP library, on the current stream or the one given; outputs and
workspaces are torch tensors of that stream, nothing synchronises, and calls can be captured into a graph.  An `out` may not overlap what is read.  There is no CPU fallback.
The calls are no part of torch's autograd: results carry no gradient function, also of inputs that require gradients, and a training step calls the gradients
itself, as below (or from a torch.autograd.Function of its own).

A training step of an experts' block, for x [T, D], w1 [E, F, D], w2 [E, D, F]:

    r = route(logits, k)                                            # R, and its entries in the order of the experts
    h = grouped_matmul(x, w1, r.expert_ptr, rows=r.token)           # [T*k, F], rows gathered from x
    y = grouped_matmul(act(h), w2, r.expert_ptr)                    # [T*k, D]
    out = combine(y, r)                                             # [T, D]
    dy, dval = combine_backward(dout, y, r)
    dh = grouped_matmul(dy, w2, r.expert_ptr, transposed=True)      # w2 the other way round
    dw2 = grouped_weight_grad(dy, act(h), r.expert_ptr)
    dw1 = grouped_weight_grad(dact(dh), x, r.expert_ptr, rows=r.token)
    dx = combine(grouped_matmul(dact(dh), w1, r.expert_ptr, transposed=True), r, weighted=False)
    dlogits = route_backward(r, dval, logits)
"""
from __future__ import annotations

import ctypes as C
from contextlib import nullcontext
from dataclasses import dataclass

from . import binding as _b
from .binding import DeviceCSR, OceanError  # noqa: F401

F32, BF16, F16 = 1, 2, 3
MAX_EXPERTS, MAX_K = 1024, 64
MAX_RANK, MAX_ADAPTERS = 256, 8192


class ocean_routing(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("experts", C.c_int64), ("k", C.c_int32), ("reserved", C.c_int32), ("row_ptr", C.c_void_p),
                ("col_idx", C.c_void_p), ("val", C.c_void_p), ("expert_ptr", C.c_void_p), ("token", C.c_void_p), ("slot", C.c_void_p)]


class ocean_groups(C.Structure):
    _fields_ = [("rows", C.c_int64), ("experts", C.c_int64), ("group_ptr", C.c_void_p), ("row_index", C.c_void_p), ("x_rows", C.c_int64)]


class ocean_adapters(C.Structure):
    _fields_ = [("adapters", C.c_int64), ("rank", C.c_int64), ("a", C.c_void_p), ("ld_a", C.c_int64), ("stride_a", C.c_int64),
                ("b", C.c_void_p), ("ld_b", C.c_int64), ("stride_b", C.c_int64), ("ranks", C.c_void_p), ("scale", C.c_void_p)]


_lib = None


def load():
    """The HIP library with the argument types of ocean_routed.h set."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _b.load()
    P, vp, i64, i32, size = C.POINTER, C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
    lib.ocean_route_workspace.argtypes = [i64, i64, i32]
    lib.ocean_route_workspace.restype = size
    lib.ocean_route.argtypes = [vp, i32, i64, i32, P(ocean_routing), vp, size, vp]
    lib.ocean_route_backward.argtypes = [P(ocean_routing), vp, vp, i32, i64, i32, vp, i64, vp]
    lib.ocean_combine.argtypes = [P(ocean_routing), vp, i32, i64, i64, vp, i64, vp]
    lib.ocean_combine_backward.argtypes = [P(ocean_routing), vp, i64, vp, i64, i32, i64, vp, i64, vp, vp]
    lib.ocean_grouped_matmul.argtypes = [P(ocean_groups), i32, i64, i64, vp, i64, vp, i64, i64, i32, vp, i64, vp]
    lib.ocean_grouped_weight_grad.argtypes = [P(ocean_groups), i32, i64, i64, vp, i64, vp, i64, vp, i64, i64, i32, vp]
    lib.ocean_adapter_workspace.argtypes = [i64, i64, i64, i64, i64, i32]
    lib.ocean_adapter_workspace.restype = size
    lib.ocean_adapter_matmul.argtypes = [P(ocean_adapters), vp, i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, size, vp]
    for name in ("ocean_route", "ocean_route_backward", "ocean_combine", "ocean_combine_backward", "ocean_grouped_matmul",
                 "ocean_grouped_weight_grad", "ocean_adapter_matmul"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


@dataclass(frozen=True)
class Routing:
    """A routing matrix in CSR (row_ptr int64 [tokens+1], col_idx int32, val float32 or None) and in the order of its columns
    (expert_ptr int64 [experts+1], token int32, slot int32).  The four entry arrays have tokens * k places; those behind the last
    entry hold -1 (val: 0)."""
    tokens: int
    experts: int
    k: int
    row_ptr: "object"
    col_idx: "object"
    val: "object"
    expert_ptr: "object"
    token: "object"
    slot: "object"

    def __post_init__(self):
        """The lists are contiguous, of their types, of their sizes and on one device."""
        import torch
        n, device = self.tokens * self.k, self.row_ptr.device
        for name, dtype, size in (("row_ptr", torch.int64, self.tokens + 1), ("col_idx", torch.int32, n), ("val", torch.float32, n),
                                  ("expert_ptr", torch.int64, self.experts + 1), ("token", torch.int32, n), ("slot", torch.int32, n)):
            t = getattr(self, name)
            if t is not None or name != "val":
                _vector(t, name, dtype, size, device)
        self._hold(device, self.val is not None)

    def _hold(self, device, weighted):
        """The C structs, with val and without, for as long as the lists are held."""
        lists = [_ptr(t) for t in (self.row_ptr, self.col_idx, self.val if weighted else None, self.expert_ptr, self.token, self.slot)]
        c = ocean_routing(self.tokens, self.experts, self.k, 0, *lists)
        lists[2] = None
        self.__dict__.update(_device=device, _structs=(ocean_routing(self.tokens, self.experts, self.k, 0, *lists), c))

    @classmethod
    def _made(cls, *fields):
        """One whose lists this module has just made."""
        r = object.__new__(cls)
        r.__dict__.update(zip(cls.__dataclass_fields__, fields))
        r._hold(r.row_ptr.device, True)
        return r

    def __reduce__(self):
        """Copies and pickles are made of the fields: the structs hold pointers to this one's lists."""
        return Routing, tuple(getattr(self, name) for name in self.__dataclass_fields__)

    def csr(self) -> DeviceCSR:
        """The matrix as an operand of binding.spgemm (without val every weight is 1); reads the number of its entries back."""
        import torch
        n = int(self.row_ptr[-1])
        val = self.val[:n] if self.val is not None else torch.ones(n, dtype=torch.float32, device=self._device)
        return DeviceCSR(self.tokens, self.experts, self.row_ptr, self.col_idx[:n], val, [self])

    def _struct(self, weighted=True):
        return self._structs[bool(weighted)]

    def _lists(self, device):
        if device != self._device:
            raise ValueError(f"the routing is on {self._device}, not {device}")
        return self.row_ptr, self.col_idx, self.val, self.expert_ptr, self.token, self.slot


# ---------------------------------------------------------------- arguments
_codes = {}


def _code(dtype) -> int:
    if not _codes:
        torch = _b._torch()
        _codes.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _codes.get(dtype)
    if code is None:
        raise TypeError(f"{dtype}: matrices are float32, bfloat16 or float16")
    return code


def _ptr(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _vector(t, name, dtype, size, device):
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != size or t.device != device or (size > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {size} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _matrix(t, name, rows=None, width=None, like=None):
    """Row stride of a matrix whose rows are contiguous; rows / width / like: what it has to have."""
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or (width is not None and t.shape[1] != width):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {'width' if width is None else width}], not {tuple(t.shape)}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} is {t.dtype} on {t.device}, not {like.dtype} on {like.device}")
    n, w = t.shape
    if w > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if n <= 1:
        return max(w, 1)
    if t.stride(0) < w:
        raise ValueError(f"{name}: rows overlap")
    return max(t.stride(0), 1)


_HERE = nullcontext()
_raw_stream = None


def _at(device, stream, *tensors):
    """(the stream's pointer, the context in which it is current on `device`): tensors made inside belong to it, and those that the call
    uses and another stream made are kept until it is done with them."""
    global _raw_stream
    torch = _b._torch()
    if device.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, not {device}")
    if stream is None:
        if _raw_stream is None:   # (a fifth of the time of current_stream(), where torch has it)
            _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        return _raw_stream(device.index), _HERE if device.index == torch.cuda.current_device() else torch.cuda.device(device)
    if stream != torch.cuda.current_stream(device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
    return int(stream.cuda_stream), torch.cuda.stream(stream)


def _output(out, shape, like, name="out"):
    """The caller's output, checked, or a new one."""
    if out is None:
        return like.new_empty(shape)
    if tuple(out.shape) != tuple(shape):
        raise ValueError(f"{name} must be {tuple(shape)}, not {tuple(out.shape)}")
    return out


# ---------------------------------------------------------------- routing
def route(logits, k: int, *, normalize: bool = True, stream=None) -> Routing:
    """The routing matrix of logits [tokens, experts]: each row's k largest, ties to the lowest columns; NaN, -inf and the type's
    lowest value are never taken.  Weights: softmax over the entries taken, or (normalize=False) over all that may be."""
    import torch
    lib = load()
    ld = _matrix(logits, "logits")
    code = _code(logits.dtype)
    T, E = logits.shape
    if not 1 <= k <= min(E, MAX_K) or E > MAX_EXPERTS:
        raise ValueError(f"k must be 1 to min(experts, {MAX_K}) and experts at most {MAX_EXPERTS}, not {k} of {E}")
    dev = logits.device
    s, here = _at(dev, stream, logits)
    with here:
        n = T * k
        row_ptr, expert_ptr = torch.empty(T + E + 2, dtype=torch.int64, device=dev).split((T + 1, E + 1))
        val, col_idx, token, slot = torch.empty((4, n), dtype=torch.int32, device=dev).unbind(0)
        r = Routing._made(T, E, k, row_ptr, col_idx, val.view(torch.float32), expert_ptr, token, slot)
        nbytes = lib.ocean_route_workspace(T, E, k)
        space = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
        _b._check(lib.ocean_route(_ptr(logits), code, ld, int(normalize), C.byref(r._struct()), _ptr(space), nbytes, s))
    return r


def route_backward(routing: Routing, dval, logits, *, normalize: bool = True, out=None, stream=None):
    """Gradient of the logits from dval [tokens*k], that of the weights in the order of routing.val; normalize as in route.  Masked logits get 0."""
    import torch
    lib = load()
    ld = _matrix(logits, "logits", routing.tokens, routing.experts)
    lists = routing._lists(logits.device)
    if routing.val is None:
        raise ValueError("the routing has no weights")
    _vector(dval, "dval", torch.float32, routing.tokens * routing.k, logits.device)
    s, here = _at(logits.device, stream, logits, dval, out, *lists)
    with here:
        out = _output(out, logits.shape, logits)
        ldo = _matrix(out, "out", like=logits)
        _b._check(lib.ocean_route_backward(C.byref(routing._struct()), _ptr(dval), _ptr(logits), _code(logits.dtype), ld, int(normalize), _ptr(out), ldo, s))
    return out


def combine(y, routing: Routing, *, weighted: bool = True, out=None, stream=None):
    """out[t] = sum of val[p] * y[slot[p]] over the entries p of row t (weighted=False, or a routing without val: of y[slot[p]])."""
    lib = load()
    ldy = _matrix(y, "y", routing.tokens * routing.k)
    lists = routing._lists(y.device)
    s, here = _at(y.device, stream, y, out, *lists)
    with here:
        out = _output(out, (routing.tokens, y.shape[1]), y)
        ldo = _matrix(out, "out", like=y)
        _b._check(lib.ocean_combine(C.byref(routing._struct(weighted)), _ptr(y), _code(y.dtype), y.shape[1], ldy, _ptr(out), ldo, s))
    return out


def combine_backward(dout, y, routing: Routing, *, weighted: bool = True, stream=None):
    """(dy, dval): gradients of y and of val.  y=None: dval is not wanted, and None."""
    import torch
    lib = load()
    ldo = _matrix(dout, "dout", routing.tokens)
    width, n = dout.shape[1], routing.tokens * routing.k
    ldy = _matrix(y, "y", n, width, like=dout) if y is not None else width
    lists = routing._lists(dout.device)
    s, here = _at(dout.device, stream, dout, y, *lists)
    with here:
        dy = dout.new_empty((n, width))
        dval = torch.empty(n, dtype=torch.float32, device=dout.device) if y is not None else None
        _b._check(lib.ocean_combine_backward(C.byref(routing._struct(weighted)), _ptr(dout), ldo, _ptr(y), ldy, _code(dout.dtype), width, _ptr(dy), max(width, 1),
                                             _ptr(dval), s))
    return dy, dval


# ---------------------------------------------------------------- grouped products
def _matrices(w, name, shape=None, like=None):
    """(row stride, stride from one matrix to the next) of matrices whose rows are contiguous."""
    if w.dim() != 3 or (shape is not None and tuple(w.shape) != tuple(shape)):
        raise ValueError(f"{name} must be [experts, rows, width]{'' if shape is None else f' = {tuple(shape)}'}, not {tuple(w.shape)}")
    if like is not None and (w.dtype != like.dtype or w.device != like.device):
        raise ValueError(f"{name} is {w.dtype} on {w.device}, not {like.dtype} on {like.device}")
    n, rows, width = w.shape
    if width > 1 and w.stride(2) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if rows > 1 and w.stride(1) < width:
        raise ValueError(f"{name}: rows overlap")
    return w.stride(1) if rows > 1 else max(width, 1), w.stride(0) if n > 1 else 0


def _groups(x, expert_ptr, rows):
    import torch
    n = x.shape[0] if rows is None else rows.shape[0]
    experts = expert_ptr.numel() - 1
    _vector(expert_ptr, "expert_ptr", torch.int64, max(experts, 0) + 1, x.device)
    if rows is not None:
        _vector(rows, "rows", torch.int32, n, x.device)
    return ocean_groups(n, experts, expert_ptr.data_ptr(), _ptr(rows), x.shape[0])


def grouped_matmul(x, w, expert_ptr, *, rows=None, transposed: bool = False, out=None, stream=None):
    """y[s] = x[rows[s]] @ w[e].T for the slots s of expert e, expert_ptr[e] .. expert_ptr[e+1]-1 (int64 [experts+1]); w [experts, outer, inner].
    transposed: w is [experts, inner, outer] and y[s] = x[rows[s]] @ w[e].  rows (int32) None: slot s is row s of x; a row number
    outside x stands for zeros.  Slots of no expert give zeros.  The gradient of x's rows is grouped_matmul(dy, w, expert_ptr,
    transposed=not transposed)."""
    lib = load()
    ldx = _matrix(x, "x")
    code = _code(x.dtype)
    ldw, stride = _matrices(w, "w", like=x)
    g = _groups(x, expert_ptr, rows)
    outer, inner = (w.shape[2], w.shape[1]) if transposed else (w.shape[1], w.shape[2])
    if w.shape[0] != g.experts or inner != x.shape[1]:
        raise ValueError(f"w is {tuple(w.shape)}{' (transposed)' if transposed else ''}: not {g.experts} matrices for rows of {x.shape[1]}")
    s, here = _at(x.device, stream, x, w, expert_ptr, rows, out)
    with here:
        out = _output(out, (g.rows, outer), x)
        ldo = _matrix(out, "out", like=x)
        _b._check(lib.ocean_grouped_matmul(C.byref(g), code, inner, outer, _ptr(x), ldx, _ptr(w), ldw, stride, int(transposed), _ptr(out), ldo, s))
    return out


def grouped_weight_grad(dy, x, expert_ptr, *, rows=None, transposed: bool = False, out=None, stream=None):
    """Gradient of grouped_matmul's w: the sum over the slots s of expert e of dy[s]^T x[rows[s]], [experts, outer, inner] (transposed:
    [experts, inner, outer]); zeros for an expert without slots.  Slots whose row number is outside x add nothing, whatever dy holds there."""
    lib = load()
    ldx = _matrix(x, "x")
    code = _code(x.dtype)
    g = _groups(x, expert_ptr, rows)
    ldd = _matrix(dy, "dy", g.rows, like=x)
    inner, outer = x.shape[1], dy.shape[1]
    s, here = _at(x.device, stream, x, dy, expert_ptr, rows, out)
    with here:
        out = _output(out, (g.experts, inner, outer) if transposed else (g.experts, outer, inner), x)
        ldo, stride = _matrices(out, "out", like=x)
        _b._check(lib.ocean_grouped_weight_grad(C.byref(g), code, inner, outer, _ptr(dy), ldd, _ptr(x), ldx, _ptr(out), ldo, stride, int(transposed), s))
    return out


# ---------------------------------------------------------------- adapters
def adapter_matmul(x, w, a, b, ids, *, ranks=None, scale=None, out=None, stream=None):
    """y[m] = x[m] @ w.T + scale[i] * (x[m] @ a[i].T) @ b[i].T with i = ids[m]; x [rows, inner], w [outer, inner], a [adapters, rank, inner],
    b [adapters, outer, rank], ids int32 [rows] (outside 0 .. adapters-1: no adapter).  ranks (int32 [adapters]): only the first ranks[i]
    rows of a[i] and columns of b[i] are used.  scale: float32 [adapters], None for 1."""
    import torch
    lib = load()
    ldx = _matrix(x, "x")
    code = _code(x.dtype)
    (rows, inner), dev = x.shape, x.device
    ldw = _matrix(w, "w", width=inner, like=x)
    outer = w.shape[0]
    if a.dim() != 3 or b.dim() != 3:
        raise ValueError(f"a must be [adapters, rank, inner] and b [adapters, outer, rank], not {tuple(a.shape)} and {tuple(b.shape)}")
    adapters, rank = a.shape[:2]
    if adapters > MAX_ADAPTERS or rank > MAX_RANK:
        raise ValueError(f"at most {MAX_ADAPTERS} adapters of rank {MAX_RANK}, not {adapters} of {rank}")
    lda, sa = _matrices(a, "a", (adapters, rank, inner), x)
    ldb, sb = _matrices(b, "b", (adapters, outer, rank), x)
    _vector(ids, "ids", torch.int32, rows, dev)
    if ranks is not None:
        _vector(ranks, "ranks", torch.int32, adapters, dev)
    if scale is not None:
        _vector(scale, "scale", torch.float32, adapters, dev)
    s, here = _at(dev, stream, x, w, a, b, ids, ranks, scale, out)
    with here:
        out = _output(out, (rows, outer), x)
        ldo = _matrix(out, "out", like=x)
        nbytes = lib.ocean_adapter_workspace(rows, inner, outer, adapters, rank, code)
        space = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        c = ocean_adapters(adapters, rank, _ptr(a), lda, sa, _ptr(b), ldb, sb, _ptr(ranks), _ptr(scale))
        _b._check(lib.ocean_adapter_matmul(C.byref(c), _ptr(ids), code, rows, inner, outer, _ptr(x), ldx, _ptr(w), ldw, _ptr(out), ldo,
                                           space.data_ptr(), nbytes, s))
    return out
