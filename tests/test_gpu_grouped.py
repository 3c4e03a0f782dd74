"""Products of ragged groups (grouped_matmul, grouped_weight_grad) against their definition in 64 bits.

Tolerance: a sum of c products in 32 bits, in any order, is off by at most (c + 1) roundings of 2^-24 of the sum of their magnitudes (products of
two 16-bit numbers are exact, those in single precision one rounding more), and is then rounded to its type."""
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


def _close(got, want, mag, c, dtype):
    return bool(np.all(np.abs(_np(got) - want) <= (c + 2) * 2.0 ** -24 * mag + EPS[dtype] * np.abs(want) + TINY[dtype]))


def _rand(gen, *shape, dtype):
    import torch
    return torch.randn(*shape, generator=gen).to(getattr(torch, dtype))


def _ptr(sizes, start=0):
    import torch
    return torch.tensor(np.cumsum([start] + list(sizes)), dtype=torch.int64)


# groups of no row, one row, a tile less one / exactly / and one, and more; widths below, at and beyond a tile and a step; odd ones
CASES = [([1], 8, 8), ([0, 1, 0, 2], 64, 64), ([3], 1, 1), ([17, 0, 15, 16], 72, 40), ([127, 128, 129, 0], 136, 200), ([5, 300], 65, 130),
         ([255, 257, 1], 264, 520), ([33, 64], 1001, 67), ([600], 128, 256), ([40, 31, 2, 90, 0, 0, 7], 200, 264), ([16], 0, 24), ([0, 0], 32, 32)]


@pytest.mark.parametrize("sizes,K,N", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gather", [False, True])
def test_products_and_gradients(rt, sizes, K, N, dtype, gather):
    import torch
    g = torch.Generator().manual_seed(sum(sizes) * 7 + K + N)
    S, E, X = sum(sizes), len(sizes), max(1, sum(sizes) // 2)
    ptr = _ptr(sizes)
    rows = torch.randint(0, X, (S,), generator=g, dtype=torch.int32) if gather else None
    x = _rand(g, X if gather else S, K, dtype=dtype)
    w, dy = _rand(g, E, N, K, dtype=dtype), _rand(g, S, N, dtype=dtype)
    r = None if rows is None else rows.cuda()
    nr = None if rows is None else _np(rows)
    want, mag = O.grouped(_np(ptr), _np(x), _np(w), nr)
    got = rt.grouped_matmul(x.cuda(), w.cuda(), ptr.cuda(), rows=r)
    assert got.shape == (S, N) and _close(got, want, mag, K, dtype)
    kn = w.transpose(1, 2).contiguous()
    assert _close(rt.grouped_matmul(x.cuda(), kn.cuda(), ptr.cuda(), rows=r, transposed=True), want, mag, K, dtype)
    # gradient of the rows: the other way round
    wdx, mdx = O.grouped(_np(ptr), _np(dy), _np(w).transpose(0, 2, 1), None)
    assert _close(rt.grouped_matmul(dy.cuda(), w.cuda(), ptr.cuda(), transposed=True), wdx, mdx, N, dtype)
    assert _close(rt.grouped_matmul(dy.cuda(), kn.cuda(), ptr.cuda()), wdx, mdx, N, dtype)
    # gradient of the weights
    wdw, mdw = O.grouped_weight_grad(_np(ptr), _np(dy), _np(x), nr)
    c = max(sizes)
    assert _close(rt.grouped_weight_grad(dy.cuda(), x.cuda(), ptr.cuda(), rows=r), wdw, mdw, c, dtype)
    assert _close(rt.grouped_weight_grad(dy.cuda(), x.cuda(), ptr.cuda(), rows=r, transposed=True), wdw.transpose(0, 2, 1), mdw.transpose(0, 2, 1), c, dtype)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_rows_and_many_groups(rt, dtype):
    import torch
    g = torch.Generator().manual_seed(1)
    sizes = [int(n) for n in torch.randint(0, 60, (150,), generator=g)]
    sizes[7], sizes[100] = 700, 1100
    S, K, N = sum(sizes), 96, 320
    ptr = _ptr(sizes)
    x, w = _rand(g, S, K, dtype=dtype), _rand(g, 150, N, K, dtype=dtype)
    dy = _rand(g, S, N, dtype=dtype)
    want, mag = O.grouped(_np(ptr), _np(x), _np(w))
    assert _close(rt.grouped_matmul(x.cuda(), w.cuda(), ptr.cuda()), want, mag, K, dtype)
    wdw, mdw = O.grouped_weight_grad(_np(ptr), _np(dy), _np(x))
    assert _close(rt.grouped_weight_grad(dy.cuda(), x.cuda(), ptr.cuda()), wdw, mdw, max(sizes), dtype)


def test_large_tiles(rt):
    """Groups of several hundred rows and widths of several hundred, where the widest tiles are taken, against 64-bit products on the GPU."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    sizes, K, N = [700, 0, 513, 900], 520, 776
    ptr, S = _ptr(sizes).cuda(), sum(sizes)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        x = torch.randn(1000, K, device="cuda", generator=g).to(dtype)
        w = torch.randn(4, N, K, device="cuda", generator=g).to(dtype)
        dy = torch.randn(S, N, device="cuda", generator=g).to(dtype)
        rows = torch.randint(0, 1000, (S,), device="cuda", generator=g, dtype=torch.int32)
        got = {"y": rt.grouped_matmul(x, w, ptr, rows=rows), "t": rt.grouped_matmul(x, w.transpose(1, 2).contiguous(), ptr, rows=rows, transposed=True),
               "dx": rt.grouped_matmul(dy, w, ptr, transposed=True), "dw": rt.grouped_weight_grad(dy, x, ptr, rows=rows),
               "dt": rt.grouped_weight_grad(dy, x, ptr, rows=rows, transposed=True)}
        for e in range(4):
            lo, hi = int(ptr[e]), int(ptr[e + 1])
            xe, we, de = x[rows[lo:hi].long()].double(), w[e].double(), dy[lo:hi].double()
            for name, at, a, b in (("y", slice(lo, hi), xe, we.T), ("t", slice(lo, hi), xe, we.T), ("dx", slice(lo, hi), de, we),
                                   ("dw", e, de.T, xe), ("dt", e, xe.T, de)):
                want, mag, c = a @ b, a.abs() @ b.abs(), a.shape[1]
                assert _close(got[name][at], _np(want), _np(mag), c, str(dtype)[6:]), (name, e, dtype)


def test_rows_of_no_group_are_cleared(rt):
    import torch
    g = torch.Generator().manual_seed(3)
    x, w = _rand(g, 500, 64, dtype="bfloat16"), _rand(g, 3, 80, 64, dtype="bfloat16")
    for sizes, start in (([20, 0, 30], 40), ([0, 0, 0], 0), ([0, 0, 0], 500), ([400, 0, 30], 70), ([1, 1, 1], 0)):
        ptr = _ptr(sizes, start)
        lo, hi = start, start + sum(sizes)
        bad = x.clone()
        bad[:lo] = float("nan")
        bad[hi:] = float("inf")
        out = torch.full((500, 80), float("nan"), device="cuda", dtype=torch.bfloat16)
        rt.grouped_matmul(bad.cuda(), w.cuda(), ptr.cuda(), out=out)
        want, mag = O.grouped(_np(ptr), _np(x), _np(w))
        assert _close(out, want, mag, 64, "bfloat16") and not bool(out[:lo].any()) and not bool(out[hi:].any())
        dy = _rand(g, 500, 80, dtype="bfloat16")
        dbad = dy.clone()
        dbad[:lo] = float("inf")
        dbad[hi:] = float("nan")
        wdw, mdw = O.grouped_weight_grad(_np(ptr), _np(dy), _np(x))
        assert _close(rt.grouped_weight_grad(dbad.cuda(), bad.cuda(), ptr.cuda()), wdw, mdw, max(max(sizes), 1), "bfloat16")


def test_no_groups_and_no_rows(rt):
    import torch
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    x = torch.randn(9, 16, device="cuda")
    assert not bool(rt.grouped_matmul(x, torch.empty(0, 8, 16, device="cuda"), one).any())
    assert rt.grouped_weight_grad(torch.randn(9, 8, device="cuda"), x, one).shape == (0, 8, 16)
    none = torch.zeros(3, dtype=torch.int64, device="cuda")
    assert rt.grouped_matmul(x[:0], torch.randn(2, 8, 16, device="cuda"), none).shape == (0, 8)
    assert not bool(rt.grouped_weight_grad(torch.randn(0, 8, device="cuda"), x[:0], none).any())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_row_numbers_outside_x_stand_for_zeros(rt, dtype):
    import torch
    g = torch.Generator().manual_seed(4)
    for K, N in ((64, 72), (51, 33), (256, 512)):
        sizes = [300, 20]
        x, w, dy = _rand(g, 50, K, dtype=dtype), _rand(g, 2, N, K, dtype=dtype), _rand(g, 320, N, dtype=dtype)
        rows = torch.randint(-3, 55, (320,), generator=g, dtype=torch.int32)
        rows[5], rows[6] = 2 ** 31 - 1, -2 ** 31
        ptr = _ptr(sizes)
        want, mag = O.grouped(_np(ptr), _np(x), _np(w), _np(rows))
        got = rt.grouped_matmul(x.cuda(), w.cuda(), ptr.cuda(), rows=rows.cuda())
        assert _close(got, want, mag, K, dtype) and not bool(got[rows.cuda() < 0].any())
        wdw, mdw = O.grouped_weight_grad(_np(ptr), _np(dy), _np(x), _np(rows))
        assert _close(rt.grouped_weight_grad(dy.cuda(), x.cuda(), ptr.cuda(), rows=rows.cuda()), wdw, mdw, 300, dtype)


def test_offsets_that_make_no_sense_stay_inside(rt):
    import torch
    g = torch.Generator().manual_seed(5)
    x, w = _rand(g, 100, 64, dtype="bfloat16").cuda(), _rand(g, 3, 64, 64, dtype="bfloat16").cuda()
    guard = torch.full((300, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    for p in ([-50, 20, 10, 1 << 40], [90, 30, -1, 7], [1000, 1000, 1000, 1000], [0, 100, 100, 200]):
        ptr = torch.tensor(p, dtype=torch.int64, device="cuda")
        rt.grouped_matmul(x, w, ptr, out=guard[100:200])
        rt.grouped_weight_grad(x, x, ptr)
        assert bool((guard[:100] == 7).all()) and bool((guard[200:] == 7).all())


@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_strides_and_alignment(rt, dtype):
    import torch
    g = torch.Generator().manual_seed(6)
    sizes, K, N = [70, 3, 130], 128, 192
    S, ptr = sum(sizes), _ptr(sizes).cuda()
    x, w, dy = (_rand(g, *s, dtype=dtype).cuda() for s in ((S, K), (3, N, K), (S, N)))
    y, dw, dx = rt.grouped_matmul(x, w, ptr), rt.grouped_weight_grad(dy, x, ptr), rt.grouped_matmul(dy, w, ptr, transposed=True)

    def held(t, off, extra):
        big = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), device="cuda", dtype=t.dtype)
        big[..., off:off + t.shape[-1]] = t
        return big[..., off:off + t.shape[-1]]

    for off, extra in ((8, 64), (1, 3), (4, 12), (0, 1), (2, 66)):
        xs, ws, ds = held(x, off, extra), held(w, off, extra), held(dy, off, extra)
        out = torch.full((S, N + extra), 7.0, device="cuda", dtype=x.dtype)
        rt.grouped_matmul(xs, ws, ptr, out=out[:, off:off + N])
        # (another tile or loader adds up in another order)
        assert torch.allclose(out[:, off:off + N].float(), y.float(), rtol=2 * EPS[dtype], atol=1e-3)
        assert bool((out[:, :off] == 7).all()) and bool((out[:, off + N:] == 7).all())
        assert torch.allclose(rt.grouped_matmul(ds, ws, ptr, transposed=True).float(), dx.float(), rtol=2 * EPS[dtype], atol=1e-3)
        held_dw = torch.full((3, N, K + extra), 7.0, device="cuda", dtype=x.dtype)
        rt.grouped_weight_grad(ds, xs, ptr, out=held_dw[:, :, off:off + K])
        assert torch.allclose(held_dw[:, :, off:off + K].float(), dw.float(), rtol=2 * EPS[dtype], atol=1e-3)
        assert bool((held_dw[:, :, :off] == 7).all()) and bool((held_dw[:, :, off + K:] == 7).all())


def test_gradients_against_differences(rt):
    """In single precision, along random directions: the product is linear in each argument, so differences are exact but for rounding."""
    import torch
    g = torch.Generator().manual_seed(7)
    sizes, K, N, X = [30, 0, 41], 48, 56, 40
    ptr = _ptr(sizes).cuda()
    rows = torch.randint(0, X, (71,), generator=g, dtype=torch.int32).cuda()
    x, w, dy = (_rand(g, *s, dtype="float32").cuda() for s in ((X, K), (3, N, K), (71, N)))
    vx, vw = (_rand(g, *s, dtype="float32").cuda() for s in ((X, K), (3, N, K)))

    def loss(x_, w_):
        return float((rt.grouped_matmul(x_, w_, ptr, rows=rows).double() * dy.double()).sum())

    dslots = rt.grouped_matmul(dy, w, ptr, transposed=True)
    dx = torch.zeros(X, K, device="cuda", dtype=torch.float64).index_add_(0, rows.long(), dslots.double())
    dw = rt.grouped_weight_grad(dy, x, ptr, rows=rows)
    size = 71 * N * K   # products of three numbers of about 1; each side off by (K + 2) * 2^-24 of them at most
    assert abs((loss(x + vx, w) - loss(x - vx, w)) / 2 - float((dx * vx.double()).sum())) <= 3 * (K + 2) * 2.0 ** -24 * size
    assert abs((loss(x, w + vw) - loss(x, w - vw)) / 2 - float((dw.double() * vw.double()).sum())) <= 3 * (K + 2) * 2.0 ** -24 * size


def test_another_stream_and_a_graph(rt):
    import torch
    g = torch.Generator().manual_seed(8)
    ptr = _ptr([60, 90]).cuda()
    x, w = _rand(g, 150, 128, dtype="bfloat16").cuda(), _rand(g, 2, 128, 128, dtype="bfloat16").cuda()
    want = rt.grouped_matmul(x, w, ptr)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = rt.grouped_matmul(x, w, ptr, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = rt.grouped_matmul(x, w, ptr)
        dw = rt.grouped_weight_grad(y, x, ptr)
    for i in range(4):
        x.copy_(torch.randn(150, 128, device="cuda"))
        ptr.copy_(_ptr([10 * i, 150 - 20 * i]).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want = rt.grouped_matmul(x, w, ptr)
        assert torch.equal(y, want) and torch.equal(dw, rt.grouped_weight_grad(want, x, ptr))


def test_refusals(rt):
    import ctypes
    import torch
    x, w = torch.randn(10, 16, device="cuda"), torch.randn(2, 8, 16, device="cuda")
    ptr = torch.tensor([0, 4, 10], device="cuda")
    rows = torch.zeros(10, dtype=torch.int32, device="cuda")
    for call in (lambda: rt.grouped_matmul(x, w, ptr.int()), lambda: rt.grouped_matmul(x, w, ptr[:2]), lambda: rt.grouped_matmul(x, w, ptr.cpu()),
                 lambda: rt.grouped_matmul(x, w[:, :, :15], ptr), lambda: rt.grouped_matmul(x, w, ptr, transposed=True),
                 lambda: rt.grouped_matmul(x, w.half(), ptr), lambda: rt.grouped_matmul(x, w, ptr, rows=rows.long()), lambda: rt.grouped_matmul(x.T, w, ptr),
                 lambda: rt.grouped_matmul(x, w, ptr, out=torch.empty(9, 8, device="cuda")), lambda: rt.grouped_matmul(x, w, ptr, out=torch.empty(10, 8)),
                 lambda: rt.grouped_matmul(x, w.transpose(1, 2), ptr, transposed=True), lambda: rt.grouped_matmul(x.cpu(), w.cpu(), ptr.cpu()),
                 lambda: rt.grouped_weight_grad(x[:9], x, ptr), lambda: rt.grouped_weight_grad(x.half(), x, ptr)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        rt.grouped_matmul(x.double(), w.double(), ptr)
    lib = rt.load()
    y = torch.empty(10, 8, device="cuda")
    g = rt.ocean_groups(10, 2, ptr.data_ptr(), None, 10)
    at = [t.data_ptr() for t in (x, w, y)]

    def product(g, dtype=1, ld_x=16, ld_y=8, x=at[0], stride=128):
        return lib.ocean_grouped_matmul(ctypes.byref(g) if g else None, dtype, 16, 8, x, ld_x, at[1], 16, stride, 0, at[2], ld_y, None)

    assert product(g) == 0
    for rc, word in ((lambda: product(None), "null"), (lambda: product(g, dtype=0), "dtype"), (lambda: product(g, ld_x=15), "stride"),
                     (lambda: product(g, ld_y=7), "stride"), (lambda: product(g, x=None), "null"), (lambda: product(g, x=at[0] + 1), "aligned"),
                     (lambda: product(g, stride=-1), "stride"), (lambda: product(rt.ocean_groups(10, 2, None, None, 10)), "group_ptr"),
                     (lambda: product(rt.ocean_groups(10, 2, ptr.data_ptr(), None, 9)), "x_rows"),
                     (lambda: lib.ocean_grouped_weight_grad(ctypes.byref(g), 1, 16, 8, at[2], 8, at[0], 16, at[1], 16, 100, 0, None), "overlap")):
        assert rc() == 1 and word in lib.ocean_last_error().decode()


def test_long_sums_in_single_precision(rt):
    """The sums of 256 products are put aside.  With numbers of either sign a sum of n terms, rounded at each of them by at most 2^-24 of what it has
    come to, is off by 2^-24 sqrt(n / 2) of its size, taken over many results: 256 terms each, then c / 256 of these."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    for c in (4096, 8192, 8191):
        x, w = torch.randn(400, c, device="cuda", generator=g), torch.randn(2, 200, c, device="cuda", generator=g)
        dy, z = torch.randn(c, 136, device="cuda", generator=g), torch.randn(c, 200, device="cuda", generator=g)
        ptr, one = torch.tensor([0, 150, 400], device="cuda"), torch.tensor([0, c], device="cuda")
        want = torch.cat([x[:150].double() @ w[0].double().T, x[150:].double() @ w[1].double().T])
        dw = dy.double().T @ z.double()
        for got, ref in ((rt.grouped_matmul(x, w, ptr), want), (rt.grouped_matmul(x, w.transpose(1, 2).contiguous(), ptr, transposed=True), want),
                         (rt.grouped_weight_grad(dy, z, one)[0], dw)):
            assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -24 * (128 + c / 512) ** 0.5
