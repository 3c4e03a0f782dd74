"""The routing matrix (route, combine and their gradients) against its definition in 64 bits.

Tolerances.  Whole numbers are equal.  Weights: the difference of two 32-bit numbers, exp, a sum of at most 1024 of them (error of a
tree over 64 lanes of at most 16 each: 21 roundings) and a division: under 64 roundings of 2^-24, relative, 4e-6; the logits' own
size enters exp's argument: |x - top| * 2^-24 more, at most 104 for what does not underflow, 6.3e-6 more.  So 1.1e-5 relative, and
2^-126 absolute.  Sums of n products: n + 2 roundings of 2^-24 of the sum of magnitudes, and the rounding to the type."""
import numpy as np
import pytest

from oracle import routed as O

pytestmark = pytest.mark.gpu
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # half a unit in the last place, relative
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}


@pytest.fixture(scope="module")
def rt():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import routed
    routed.load()
    return routed


def _np(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.cpu().numpy()


def _logits(T, E, dtype, seed, kind):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, E, generator=g) * 2
    if kind == "ties":
        x = torch.randint(-1, 2, (T, E), generator=g).float() * torch.where(torch.rand(T, E, generator=g) < 0.5, 1.0, -1.0)   # (-0 and 0)
    x = x.to(dtype)
    if kind == "masked":
        u = torch.rand(T, E, generator=g)
        x[u < 0.3] = float("-inf")
        x[(u >= 0.3) & (u < 0.45)] = torch.finfo(dtype).min
        x[(u >= 0.45) & (u < 0.55)] = float("nan")
        x[(u >= 0.55) & (u < 0.58)] = float("inf")
        x[(u >= 0.58) & (u < 0.6)] = torch.finfo(dtype).max
        x[::5] = torch.finfo(dtype).min
        x[1::7] = float("-inf")
        x[2::11] = float("nan")
    return x


SHAPES = [(1, 1, 1), (1, 8, 2), (3, 5, 5), (64, 64, 4), (65, 65, 8), (130, 128, 6), (777, 100, 8), (500, 257, 3), (200, 1000, 64), (0, 8, 2)]


@pytest.mark.parametrize("T,E,k", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked"])
def test_routing_matrix_and_gradient(rt, T, E, k, dtype, kind):
    import torch
    x = _logits(T, E, getattr(torch, dtype), T * 31 + E + k, kind)
    lowest = float(torch.finfo(x.dtype).min)
    for normalize in (True, False):
        ref = O.route(_np(x), k, normalize, lowest)
        r = rt.route(x.cuda(), k, normalize=normalize)
        for name in ("row_ptr", "col_idx", "expert_ptr", "token", "slot"):
            assert np.array_equal(_np(getattr(r, name)), ref[name]), name
        val = _np(r.val)
        assert np.all(np.abs(val - ref["val"]) <= 1.1e-5 * ref["val"] + 2.0 ** -126)
        dval = torch.randn(T * k, generator=torch.Generator().manual_seed(3))
        got = _np(rt.route_backward(r, dval.cuda(), x.cuda(), normalize=normalize))
        want = O.route_backward(ref, _np(dval), normalize)
        g = np.zeros((T, E))
        for t in range(T):
            for p in range(ref["row_ptr"][t], ref["row_ptr"][t + 1]):
                g[t, ref["col_idx"][p]] = abs(float(dval[p]))
        mag = ref["prob"] * (g + (ref["prob"] * g).sum(1, keepdims=True))
        assert np.all(np.abs(got - want) <= 3.5e-5 * mag + EPS[dtype] * np.abs(want) + TINY[dtype] + 2.0 ** -126)   # three factors of 1.1e-5 each


@pytest.mark.parametrize("normalize", [True, False])
def test_gradient_of_the_logits_against_differences(rt, normalize):
    import torch
    T, E, k, h = 6, 12, 4, 2.0 ** -7
    x = torch.randn(T, E, generator=torch.Generator().manual_seed(5))
    x = (torch.argsort(torch.argsort(x, 1), 1).float() - 6) * 0.25   # neighbours further apart than 2 h: no change of what is taken
    dval = torch.randn(T * k, generator=torch.Generator().manual_seed(6)).cuda()
    r = rt.route(x.cuda(), k, normalize=normalize)
    got = _np(rt.route_backward(r, dval, x.cuda(), normalize=normalize))

    def loss(y):
        return (rt.route(y.cuda(), k, normalize=normalize).val * dval).reshape(T, k).sum(1)

    for e in range(E):
        step = torch.zeros(T, E)
        step[:, e] = h
        diff = _np((loss(x + step) - loss(x - step)) / (2 * h))
        # third derivative of a softmax weight is at most 1, times h^2 / 6 and sum |dval| <= 12; rounding of the weights 1.1e-5 / h
        assert np.all(np.abs(diff - got[:, e]) <= 12 * h * h / 6 + 12 * 1.1e-5 / h)


def test_one_block_and_several(rt):
    """Up to 64 tokens take another way than more: their matrix is the same as that of the same rows among more."""
    import torch
    for T, E, k in ((64, 40, 3), (64, 300, 9), (63, 700, 20)):
        x = _logits(T, E, torch.float32, E, "masked").cuda()
        few, many = rt.route(x, k, normalize=False), rt.route(torch.cat([x, x]), k, normalize=False)
        n = int(few.row_ptr[-1])
        assert torch.equal(few.row_ptr, many.row_ptr[:T + 1]) and torch.equal(few.col_idx[:n], many.col_idx[:n]) and torch.equal(few.val[:n], many.val[:n])


def test_strided_logits_streams_and_out(rt):
    import torch
    base = torch.randn(70, 40, device="cuda")
    x = base[::2, 3:23]
    ref = O.route(_np(x), 3, True, float(torch.finfo(torch.float32).min))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r = rt.route(x, 3, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert np.array_equal(_np(r.slot), ref["slot"]) and np.array_equal(_np(r.col_idx), ref["col_idx"])
    out = torch.full((35, 64), 7.0, device="cuda")
    rt.route_backward(r, torch.ones(105, device="cuda"), x, normalize=False, out=out[:, 5:25])
    assert bool((out[:, :5] == 7).all()) and bool((out[:, 25:] == 7).all()) and not bool((out[:, 5:25] == 7).any())


@pytest.mark.parametrize("T,E,k,D", [(1, 2, 1, 1), (1, 4, 2, 4096), (37, 16, 2, 2047), (130, 9, 3, 514), (65, 8, 8, 260), (300, 16, 4, 1032), (0, 4, 2, 16), (5, 4, 2, 0)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("masked", [False, True])
def test_combine_and_gradients(rt, T, E, k, D, dtype, masked):
    import torch
    x = _logits(T, E, torch.float32, T + D, "masked" if masked else "plain")
    r = rt.route(x.cuda(), k)
    n = int(r.row_ptr[-1])
    g = torch.Generator().manual_seed(T)
    y = torch.randn(T * k, D, generator=g).to(getattr(torch, dtype))
    y[n:] = float("nan")                                  # rows that no entry names
    dout = torch.randn(T, D, generator=g).to(y.dtype)
    ptr, slot, val = _np(r.row_ptr), _np(r.slot), _np(r.val)
    y64 = np.nan_to_num(_np(y))
    for weighted in (True, False):
        v = val if weighted else np.ones_like(val)
        want, mag = O.combine(ptr, slot, v, y64)
        got = _np(rt.combine(y.cuda(), r, weighted=weighted))
        assert np.all(np.abs(got - want) <= (k + 2) * 2.0 ** -24 * mag + EPS[dtype] * np.abs(want) + TINY[dtype])
        dy, dval = rt.combine_backward(dout.cuda(), y.cuda(), r, weighted=weighted)
        wdy, wdval, dmag = O.combine_backward(ptr, slot, v, _np(dout), y64)
        assert np.all(np.abs(_np(dy) - wdy) <= (2.0 ** -23 + EPS[dtype]) * np.abs(wdy) + TINY[dtype])
        # a lane adds up a 64th of the width (two roundings a product), then the lanes
        assert np.all(np.abs(_np(dval) - wdval) <= (D / 32 + 40) * 2.0 ** -24 * dmag)
        only, none = rt.combine_backward(dout.cuda(), None, r, weighted=weighted)
        assert none is None and torch.equal(only, dy)


def test_combine_strides_and_alignment(rt):
    import torch
    T, E, k, D = 50, 8, 3, 96
    r = rt.route(_logits(T, E, torch.float32, 1, "plain").cuda(), k)
    y = torch.randn(T * k, D, device="cuda").to(torch.bfloat16)
    want = rt.combine(y, r)
    for off, ld in ((0, D), (8, 128), (1, 99), (2, 102), (4, 100)):
        held = torch.full((T * k, ld + 16), float("nan"), device="cuda", dtype=torch.bfloat16)
        held[:, off:off + D] = y
        out = torch.full((T, ld + 16), 7.0, device="cuda", dtype=torch.bfloat16)
        rt.combine(held[:, off:off + D], r, out=out[:, off:off + D])
        assert torch.equal(out[:, off:off + D], want)
        assert bool((out[:, :off] == 7).all()) and bool((out[:, off + D:] == 7).all())


def test_entries_outside_the_rows_add_nothing(rt):
    import torch
    r = rt.route(_logits(9, 4, torch.float32, 2, "plain").cuda(), 2)
    y = torch.randn(18, 32, device="cuda")
    r.slot[4] = -3
    r.slot[7] = 18
    r.row_ptr[9] = 1000                      # (beyond the arrays: limited to them)
    val = r.val.clone()
    ptr, slot = _np(r.row_ptr).clip(0, 18), _np(r.slot).copy()
    v = _np(val)
    v[4] = v[7] = 0
    slot[4] = slot[7] = 0
    want, _ = O.combine(ptr, slot, v, _np(y))
    assert np.allclose(_np(rt.combine(y, r)), want, rtol=0, atol=1e-5)


def test_product_of_the_routing_matrix_with_itself(rt):
    """R^T R over the library's sparse product: how often two experts are used together."""
    import torch
    from paper_2604_19004_amd import binding as ob
    T, E, k = 400, 24, 3
    r = rt.route(_logits(T, E, torch.float32, 4, "masked").cuda(), k)
    R = r.csr()
    ones = ob.DeviceCSR(R.rows, R.cols, R.row_ptr, R.col_idx, torch.ones_like(R.val))
    Rt = ob.DeviceCSR(E, T, r.expert_ptr, r.token[:R.nnz], torch.ones_like(R.val))
    C, _ = ob.spgemm(Rt, ones)
    dense = np.zeros((T, E))
    for t in range(T):
        dense[t, _np(R.col_idx)[_np(R.row_ptr)[t]:_np(R.row_ptr)[t + 1]]] = 1
    got = np.zeros((E, E))
    cp, cc, cv = _np(C.row_ptr), _np(C.col_idx), _np(C.val)
    for i in range(E):
        got[i, cc[cp[i]:cp[i + 1]]] = cv[cp[i]:cp[i + 1]]
    assert np.array_equal(got, dense.T @ dense)


def test_captured_into_a_graph(rt):
    """Replayed several times, with other work in between, on logits that change."""
    import torch
    T, E, k, D = 200, 32, 4, 128
    x = torch.randn(T, E, device="cuda")
    y = torch.randn(T * k, D, device="cuda").to(torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        rt.combine(y, rt.route(x, k))
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = rt.route(x, k)
        out = rt.combine(y, r)
        dy, dval = rt.combine_backward(out, y, r)
        dx = rt.route_backward(r, dval, x)
    for i in range(4):
        x.copy_(torch.randn(T, E, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        r2 = rt.route(x, k)
        out2 = rt.combine(y, r2)
        dy2, dval2 = rt.combine_backward(out2, y, r2)
        for a, b in ((r.col_idx, r2.col_idx), (r.val, r2.val), (r.slot, r2.slot), (r.expert_ptr, r2.expert_ptr), (out, out2), (dy, dy2),
                     (dval, dval2), (dx, rt.route_backward(r2, dval2, x))):
            assert torch.equal(a, b)


def test_refusals(rt):
    import torch
    x = torch.randn(8, 6, device="cuda")
    r = rt.route(x, 2)
    y = torch.randn(16, 32, device="cuda")
    for call in (lambda: rt.route(x, 0), lambda: rt.route(x, 7), lambda: rt.route(torch.randn(2, 1025, device="cuda"), 2), lambda: rt.route(x.T, 2),
                 lambda: rt.route(x[0], 2), lambda: rt.route(torch.randn(8, 6), 2), lambda: rt.combine(y[:15], r), lambda: rt.combine(y.T, r),
                 lambda: rt.combine(y, r, out=y[:8].to(torch.float16)), lambda: rt.combine(y, r, out=y[:7]),
                 lambda: rt.combine_backward(y[:8], y[:, :16], r), lambda: rt.route_backward(r, r.val[:3], x),
                 lambda: rt.route_backward(r, r.val, x[:, :5]), lambda: rt.combine(y.cpu(), r)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: rt.route(x.double(), 2), lambda: rt.combine(y.double(), r)):
        with pytest.raises(TypeError):
            call()
    import ctypes
    from paper_2604_19004_amd import binding
    x = torch.randn(200, 6, device="cuda")   # (few tokens need no workspace)
    lib, c, few = rt.load(), rt.route(x, 2)._struct(), r._struct()
    assert lib.ocean_route_workspace(8, 6, 2) == 0
    need = lib.ocean_route_workspace(200, 6, 2)
    space = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    at = space.data_ptr()
    for rc, word in ((lambda: lib.ocean_route(x.data_ptr(), 0, 6, 1, ctypes.byref(c), at, need, None), "dtype"),
                     (lambda: lib.ocean_route(x.data_ptr(), 1, 6, 1, ctypes.byref(c), at, need - 1, None), "workspace"),
                     (lambda: lib.ocean_route(x.data_ptr(), 1, 6, 1, ctypes.byref(c), at + 4, need, None), "workspace"),
                     (lambda: lib.ocean_route(x.data_ptr(), 1, 6, 1, ctypes.byref(c), None, need, None), "workspace"),
                     (lambda: lib.ocean_route(x.data_ptr(), 1, 5, 1, ctypes.byref(c), at, need, None), "stride"),
                     (lambda: lib.ocean_route(x.data_ptr() + 2, 1, 6, 1, ctypes.byref(c), at, need, None), "aligned"),
                     (lambda: lib.ocean_route(None, 1, 6, 1, ctypes.byref(c), at, need, None), "null"),
                     (lambda: lib.ocean_combine(None, y.data_ptr(), 1, 32, 32, y.data_ptr(), 32, None), "routing is null")):
        assert rc() == 1 and word in lib.ocean_last_error().decode()
    few.k = 7
    assert lib.ocean_combine(ctypes.byref(few), y.data_ptr(), 1, 32, 32, y.data_ptr(), 32, None) == 1
    assert lib.ocean_route_workspace(-1, 6, 2) == 0


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("E", [40, 700])
def test_masked_logits_get_no_gradient_whatever_that_of_the_weights_is(rt, E, normalize):
    """Gradients of weights that overflowed reach a row's open logits, not its masked ones, and no other row."""
    import torch
    T, k = 90, 3
    x = _logits(T, E, torch.float32, 7, "masked").cuda()
    lowest = torch.finfo(torch.float32).min
    masked = x.isnan() | (x <= lowest)
    for bad in (float("nan"), float("inf"), float("-inf")):
        r = rt.route(x, k, normalize=normalize)
        dval = torch.randn(T * k, generator=torch.Generator().manual_seed(3)).cuda()
        clean = rt.route_backward(r, dval, x, normalize=normalize)
        ptr = r.row_ptr.tolist()
        hit = [t for t in range(T) if ptr[t + 1] > ptr[t]][::4]
        for t in hit:
            dval[ptr[t]] = bad
        got = rt.route_backward(r, dval, x, normalize=normalize)
        assert not bool(got[masked].any())
        rest = torch.ones(T, dtype=torch.bool)
        rest[hit] = False
        assert torch.equal(got[rest.cuda()], clean[rest.cuda()]) and not bool(got[hit].isfinite().all(1).any())
