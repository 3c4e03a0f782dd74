"""Products of ragged groups with matrices in four bits (grouped_matmul_mx4) against their definition in 64 bits.

Tolerance: a sum of c products in 32 bits, in any order, is off by at most (c + 2) roundings of 2^-24 of the sum of their magnitudes, and is rounded
once to its type.  Numbers of four bits times bfloat16 numbers (or numbers of four bits) are exact products; float16 and single precision numbers
are 2 and 3 such, so there are that many times as many terms."""
import numpy as np
import pytest

from oracle import experts as X
from oracle import routed as O

pytestmark = pytest.mark.gpu
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}
TERMS = {"float32": 3, "bfloat16": 1, "float16": 2}


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts
    experts.load()
    return experts


def _np(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.cpu().numpy()


def _close(got, want, mag, c, dtype, terms=None):
    return bool(np.all(np.abs(_np(got) - want) <= (terms or TERMS[dtype]) * (c + 2) * 2.0 ** -24 * mag + EPS[dtype] * np.abs(want) + TINY[dtype]))


def _rand(gen, *shape, dtype):
    import torch
    return torch.randn(*shape, generator=gen).to(getattr(torch, dtype))


def _ptr(sizes, start=0):
    import torch
    return torch.tensor(np.cumsum([start] + list(sizes)), dtype=torch.int64)


def _four(ex, gen, *shape, spread=3, pitch=0):
    """A random matrix in four bits: every code, scales that differ by block, codes behind the end and scales behind the blocks as they fall; and its numbers."""
    import torch
    inner = shape[-1]
    blocks = (inner + 31) // 32
    codes = torch.randint(0, 256, (*shape[:-1], blocks * 16), generator=gen).to(torch.uint8)
    scales = torch.randint(0, 256, (*shape[:-1], (blocks + 15) // 16 * 16 + pitch), generator=gen).to(torch.uint8)
    scales[..., :blocks] = (127 - spread + torch.randint(0, 2 * spread + 1, (*shape[:-1], blocks), generator=gen)).to(torch.uint8)
    return ex.Mx4(codes.cuda(), scales.cuda(), inner), X.values(X.unpack(codes.numpy()), scales[..., :blocks].numpy().astype(np.int64), inner)


# groups of no row, one row, a tile less one / exactly / and one, and more; widths below, at and beyond a block, a tile and a step; odd ones
CASES = [([1], 8, 8), ([0, 1, 0, 2], 64, 64), ([3], 1, 1), ([17, 0, 15, 16], 72, 40), ([127, 128, 129, 0], 136, 200), ([5, 300], 65, 130),
         ([255, 257, 1], 264, 520), ([33, 64], 1001, 67), ([600], 128, 256), ([40, 31, 2, 90, 0, 0, 7], 200, 264), ([16], 0, 24), ([0, 0], 32, 32),
         ([2, 20, 9], 513, 33), ([70], 31, 95)]


@pytest.mark.parametrize("sizes,K,N", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gather", [False, True])
def test_products_and_the_gradient_of_rows(ex, sizes, K, N, dtype, gather):
    import torch
    g = torch.Generator().manual_seed(sum(sizes) * 7 + K + N)
    S, E, R = sum(sizes), len(sizes), max(1, sum(sizes) // 2)
    ptr = _ptr(sizes)
    rows = torch.randint(0, R, (S,), generator=g, dtype=torch.int32) if gather else None
    x, dy = _rand(g, R if gather else S, K, dtype=dtype), _rand(g, S, N, dtype=dtype)
    w, value = _four(ex, g, E, N, K)
    r = None if rows is None else rows.cuda()
    nr = None if rows is None else _np(rows)
    want, mag = O.grouped(_np(ptr), _np(x), value, nr)
    got = ex.grouped_matmul_mx4(x.cuda(), w, ptr.cuda(), rows=r)
    assert got.dtype == x.dtype and got.shape == (S, N) and _close(got, want, mag, K, dtype)
    wdx, mdx = O.grouped(_np(ptr), _np(dy), value.transpose(0, 2, 1), None)
    assert _close(ex.grouped_matmul_mx4(dy.cuda(), w, ptr.cuda(), transposed=True), wdx, mdx, N, dtype)
    # rows in four bits
    q, qvalue = _four(ex, g, R if gather else S, K)
    want, mag = O.grouped(_np(ptr), qvalue, value, nr)
    got = ex.grouped_matmul_mx4(q, w, ptr.cuda(), rows=r, dtype=x.dtype)
    assert got.dtype == x.dtype and got.shape == (S, N) and _close(got, want, mag, K, dtype, 1)


def _compare(ex, sizes, K, N, dtype, seed, rows_of_x=None, spread=3):
    """All three products against 64-bit ones on the GPU."""
    import torch
    g = torch.Generator().manual_seed(seed)
    S, E = sum(sizes), len(sizes)
    ptr = _ptr(sizes).cuda()
    R = rows_of_x or S
    rows = torch.randint(0, R, (S,), generator=g, dtype=torch.int32).cuda() if rows_of_x else None
    x, dy = _rand(g, R, K, dtype=dtype).cuda(), _rand(g, S, N, dtype=dtype).cuda()
    w, value = _four(ex, g, E, N, K, spread=spread)
    q, qvalue = _four(ex, g, R, K, spread=spread)
    value, qvalue = torch.from_numpy(value).cuda(), torch.from_numpy(qvalue).cuda()
    got = {"y": ex.grouped_matmul_mx4(x, w, ptr, rows=rows), "dx": ex.grouped_matmul_mx4(dy, w, ptr, transposed=True),
           "q": ex.grouped_matmul_mx4(q, w, ptr, rows=rows, dtype=x.dtype)}
    for e in range(E):
        lo, hi = int(ptr[e]), int(ptr[e + 1])
        if lo == hi:
            continue
        at = rows[lo:hi].long() if rows is not None else slice(lo, hi)
        for name, a, b, terms in (("y", x[at].double(), value[e].T, None), ("dx", dy[lo:hi].double(), value[e], None), ("q", qvalue[at], value[e].T, 1)):
            want, mag = a @ b, a.abs() @ b.abs()
            assert _close(got[name][lo:hi], _np(want), _np(mag), a.shape[1], dtype, terms), (name, e)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_large_tiles(ex, dtype):
    _compare(ex, [700, 0, 513, 900], 520, 776, dtype, 2, rows_of_x=1000)
    _compare(ex, [3000, 3100, 2900, 3300], 96, 2304, dtype, 3)
    _compare(ex, [2300, 4000, 2900], 257, 2500, dtype, 4, rows_of_x=4000)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_many_groups(ex, dtype):
    import torch
    g = torch.Generator().manual_seed(1)
    sizes = [int(n) for n in torch.randint(0, 60, (150,), generator=g)]
    sizes[7], sizes[100] = 700, 1100
    _compare(ex, sizes, 96, 320, dtype, 5)
    _compare(ex, [1] * 70 + [0] * 30 + [2] * 9, 160, 130, dtype, 6, rows_of_x=11)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_long_rows(ex, dtype):
    """Rows of many steps, with an end that is no whole one."""
    for K in (4096, 8192 + 37):
        _compare(ex, [3, 0, 19, 40], K, 80, dtype, K)
        _compare(ex, [130], K, 300, dtype, K + 1)
    _compare(ex, [5, 6], 200, 5001, dtype, 9)


def test_long_sums_in_single_precision(ex):
    """With numbers of either sign a sum of n terms, rounded at each of them by at most 2^-24 of what it has come to, is off by 2^-24 sqrt(n / 2) of its
    size, taken over many results: three times 256 terms each in tiles, then c / 256 of these, and in few rows an eighth of three times c."""
    import torch
    g = torch.Generator().manual_seed(6)
    for c in (4096, 8192, 8191):
        w, value = _four(ex, g, 2, 200, c)
        x = _rand(g, 400, c, dtype="float32").cuda()
        value = torch.from_numpy(value).cuda()
        for sizes in ([150, 250], [10, 9]):
            n = sum(sizes)
            want = torch.cat([x[:sizes[0]].double() @ value[0].T, x[sizes[0]:n].double() @ value[1].T])
            got = ex.grouped_matmul_mx4(x[:n], w, _ptr(sizes).cuda())
            assert float((got.double() - want).norm() / want.norm()) <= 2.0 ** -24 * (max(384, 3 * c / 16) + c / 512) ** 0.5


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_scales_far_apart(ex, dtype):
    """Numbers of four bits from 2^-60 to 2^60 beside each other, beyond what float16 has."""
    import torch
    g = torch.Generator().manual_seed(8)
    for sizes, K, N in (([5, 18], 224, 72), ([300, 290], 224, 600)):
        ptr, S = _ptr(sizes), sum(sizes)
        w, value = _four(ex, g, 2, N, K, spread=60)
        q, qvalue = _four(ex, g, S, K, spread=60)
        x, dy = _rand(g, S, K, dtype=dtype), _rand(g, S, N, dtype=dtype)
        if dtype == "float16":   # (results that float16 has: what meets the large numbers is 0)
            big = torch.from_numpy((np.abs(value).max(1) > 64)[0] | (np.abs(value).max(1) > 64)[1])
            x[:, big] = 0
            big = torch.from_numpy((np.abs(value).max(2) > 64)[0] | (np.abs(value).max(2) > 64)[1])
            dy[:, big] = 0
        out = "float32" if dtype == "float16" else dtype
        want, mag = O.grouped(_np(ptr), _np(x), value)
        assert _close(ex.grouped_matmul_mx4(x.cuda(), w, ptr.cuda()), want, mag, K, dtype)
        want, mag = O.grouped(_np(ptr), _np(dy), value.transpose(0, 2, 1))
        assert _close(ex.grouped_matmul_mx4(dy.cuda(), w, ptr.cuda(), transposed=True), want, mag, N, dtype)
        want, mag = O.grouped(_np(ptr), qvalue, value)
        assert _close(ex.grouped_matmul_mx4(q, w, ptr.cuda(), dtype=getattr(torch, out)), want, mag, K, out, 1)


def test_small_inner_products_beside_large_ones(ex):
    """float16: blocks of large numbers, met by zeros, beside small ones that make the result."""
    import torch
    g = torch.Generator().manual_seed(9)
    for sizes, N in (([4], 40), ([300], 300)):
        codes = torch.randint(0, 256, (1, N, 64), generator=g).to(torch.uint8)
        scales = torch.full((1, N, 16), 127, dtype=torch.uint8)
        scales[:, :, 0], scales[:, :, 1], scales[:, :, 2] = 160, 100, 80
        w, value = ex.Mx4(codes.cuda(), scales.cuda(), 128), X.values(X.unpack(codes.numpy()), scales[..., :4].numpy().astype(np.int64), 128)
        x = _rand(g, sum(sizes), 128, dtype="float16")
        x[:, :32], x[:, 96:] = 0, 0
        x[:, 32:64] *= 1000
        want, mag = O.grouped(_np(_ptr(sizes)), _np(x), value)
        assert _close(ex.grouped_matmul_mx4(x.cuda(), w, _ptr(sizes).cuda()), want, mag, 128, "float16")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_infinite_numbers_and_nan(ex, dtype):
    """x's, and blocks of NaN: they reach the results whose sums they are in, and no others."""
    import torch
    g = torch.Generator().manual_seed(10)
    for sizes, K, N in (([3, 20], 200, 70), ([200, 333], 200, 300)):
        S, ptr = sum(sizes), _ptr(sizes).cuda()
        x = _rand(g, S, K, dtype=dtype)
        w, value = _four(ex, g, 2, N, K)
        w.codes[w.codes % 8 == 0] += 1                    # (no zeros: an infinite number times each is infinite)
        w.codes[w.codes // 16 % 8 == 0] += 16
        w.scales[0, 5, 1], w.scales[1, 69, 6] = 255, 255
        x[2, 100], x[4, 3], x[S - 1, K - 1] = float("inf"), float("nan"), float("-inf")
        value = X.values(X.unpack(w.codes.cpu().numpy()), w.scales[..., :7].cpu().numpy().astype(np.int64), K)
        y = _np(ex.grouped_matmul_mx4(x.cuda(), w, ptr))
        with np.errstate(invalid="ignore"):
            want = np.concatenate([_np(x)[:sizes[0]] @ value[0].T, _np(x)[sizes[0]:] @ value[1].T])
        assert np.array_equal(np.isnan(y), np.isnan(want)) and np.array_equal(np.isinf(y), np.isinf(want)) and np.array_equal(y[np.isinf(y)], want[np.isinf(want)])
        q = ex.mx4_quantize(x.cuda())
        y = _np(ex.grouped_matmul_mx4(q, w, ptr, dtype=torch.float32))
        bad = np.zeros((S, N), bool)
        bad[[2, 4, S - 1]] = True
        bad[:sizes[0], 5] = True
        bad[sizes[0]:, 69] = True
        assert np.array_equal(np.isnan(y), bad)
        dy = _rand(g, S, N, dtype=dtype)
        dy[1, 9] = float("nan")
        dx = _np(ex.grouped_matmul_mx4(dy.cuda(), w, ptr, transposed=True))
        bad = np.zeros((S, K), bool)
        bad[1] = True
        bad[:sizes[0], 32:64] = True
        bad[sizes[0]:, 192:] = True
        assert np.array_equal(np.isnan(dx), bad)


def test_rows_of_no_group_are_cleared(ex):
    import torch
    g = torch.Generator().manual_seed(3)
    x = _rand(g, 500, 64, dtype="bfloat16")
    w, value = _four(ex, g, 3, 96, 64)
    for sizes, start in (([20, 0, 30], 40), ([0, 0, 0], 0), ([0, 0, 0], 500), ([400, 0, 30], 70), ([1, 1, 1], 0)):
        ptr = _ptr(sizes, start)
        lo, hi = start, start + sum(sizes)
        bad = x.clone()
        bad[:lo] = float("nan")
        bad[hi:] = float("inf")
        want, mag = O.grouped(_np(ptr), _np(x), value)
        out = torch.full((500, 96), float("nan"), device="cuda", dtype=torch.bfloat16)
        ex.grouped_matmul_mx4(bad.cuda(), w, ptr.cuda(), out=out)
        assert _close(out, want, mag, 64, "bfloat16") and not bool(out[:lo].any()) and not bool(out[hi:].any())
        out = torch.full((500, 96), float("nan"), device="cuda", dtype=torch.float16)
        ex.grouped_matmul_mx4(ex.mx4_quantize(bad.cuda()), w, ptr.cuda(), out=out)
        assert not bool(out[:lo].any()) and not bool(out[hi:].any()) and not bool(out.isnan().any())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_row_numbers_outside_x_stand_for_zeros(ex, dtype):
    import torch
    g = torch.Generator().manual_seed(4)
    for K, N, sizes in ((64, 72, [300, 20]), (51, 33, [12, 8]), (256, 512, [300, 20])):
        S = sum(sizes)
        x = _rand(g, 50, K, dtype=dtype)
        w, value = _four(ex, g, 2, N, K)
        w.scales[0, 3, 0] = 255   # (0 also where the matrix holds NaN)
        rows = torch.randint(-3, 55, (S,), generator=g, dtype=torch.int32)
        rows[5], rows[6], rows[7] = 2 ** 31 - 1, -2 ** 31, 4
        want, mag = O.grouped(_np(_ptr(sizes)), _np(x), np.where(np.isnan(value), 0, value), _np(rows))
        out = ((_np(rows) < 0) | (_np(rows) >= 50))[:, None] | np.zeros((1, N), bool)
        for y in (ex.grouped_matmul_mx4(x.cuda(), w, _ptr(sizes).cuda(), rows=rows.cuda()),
                  ex.grouped_matmul_mx4(ex.mx4_quantize(x.cuda()), w, _ptr(sizes).cuda(), rows=rows.cuda(), dtype=x.dtype)):
            y = _np(y)
            assert not y[out].any() and np.isnan(y[:sizes[0], 3][~out[:sizes[0], 3]]).all()
        y = ex.grouped_matmul_mx4(x.cuda(), w, _ptr(sizes).cuda(), rows=rows.cuda())
        y[:sizes[0], 3], want[:sizes[0], 3] = 0, 0
        assert _close(y, want, mag, K, dtype)


def test_offsets_that_make_no_sense_stay_inside(ex):
    import torch
    g = torch.Generator().manual_seed(5)
    x = _rand(g, 100, 64, dtype="bfloat16").cuda()
    w, _ = _four(ex, g, 3, 64, 64)
    guard = torch.full((300, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    for p in ([-50, 20, 10, 1 << 40], [90, 30, -1, 7], [1000, 1000, 1000, 1000], [0, 100, 100, 200]):
        ptr = torch.tensor(p, dtype=torch.int64, device="cuda")
        ex.grouped_matmul_mx4(x, w, ptr, out=guard[100:200])
        ex.grouped_matmul_mx4(x, w, ptr, out=guard[100:200], transposed=True)
        ex.grouped_matmul_mx4(ex.mx4_quantize(x), w, ptr, out=guard[100:200])
        assert bool((guard[:100] == 7).all()) and bool((guard[200:] == 7).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_strides_and_alignment(ex, dtype):
    import torch
    g = torch.Generator().manual_seed(6)
    for sizes in ([70, 3, 130], [7, 3, 13]):
        S, K, N, ptr = sum(sizes), 136, 192, _ptr(sizes).cuda()
        x, dy = _rand(g, S, K, dtype=dtype).cuda(), _rand(g, S, N, dtype=dtype).cuda()
        w, value = _four(ex, g, 3, N, K)
        want, mag = O.grouped(_np(ptr), _np(x), value)
        wdx, mdx = O.grouped(_np(ptr), _np(dy), value.transpose(0, 2, 1))

        def held(t, off, extra):
            big = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), device="cuda", dtype=t.dtype)
            big[..., off:off + t.shape[-1]] = t
            return big[..., off:off + t.shape[-1]]

        codes = torch.full((3, N + 2, 16 * 7), 255, dtype=torch.uint8, device="cuda")
        scales = torch.full((3, N + 1, 48), 255, dtype=torch.uint8, device="cuda")
        codes[:, 1:-1, 16:96], scales[:, 1:, 16:32] = w.codes, w.scales
        v = ex.Mx4(codes[:, 1:-1, 16:96], scales[:, 1:, 16:32], K)
        for off, extra in ((8, 64), (1, 3), (4, 12), (0, 1), (2, 66)):
            out = torch.full((S, N + extra), 7.0, device="cuda", dtype=x.dtype)
            ex.grouped_matmul_mx4(held(x, off, extra), v, ptr, out=out[:, off:off + N])
            assert _close(out[:, off:off + N], want, mag, K, dtype) and bool((out[:, :off] == 7).all()) and bool((out[:, off + N:] == 7).all())
            assert _close(ex.grouped_matmul_mx4(held(dy, off, extra), v, ptr, transposed=True), wdx, mdx, N, dtype)


def test_gradient_against_differences(ex):
    """The product is linear in the rows, so differences are exact but for rounding."""
    import torch
    g = torch.Generator().manual_seed(7)
    sizes, K, N, R = [30, 0, 41], 48, 56, 40
    ptr = _ptr(sizes).cuda()
    rows = torch.randint(0, R, (71,), generator=g, dtype=torch.int32).cuda()
    x, v, dy = (_rand(g, *s, dtype="float32").cuda() for s in ((R, K), (R, K), (71, N)))
    w, value = _four(ex, g, 3, N, K, spread=1)

    def loss(x_):
        return float((ex.grouped_matmul_mx4(x_, w, ptr, rows=rows).double() * dy.double()).sum())

    dx = torch.zeros(R, K, device="cuda", dtype=torch.float64).index_add_(0, rows.long(), ex.grouped_matmul_mx4(dy, w, ptr, transposed=True).double())
    size = 71 * N * K * float(np.abs(value).mean()) * 2   # each side off by 3 (K + 2) * 2^-24 of the magnitudes at most
    assert abs((loss(x + v) - loss(x - v)) / 2 - float((dx * v.double()).sum())) <= 9 * (K + 2) * 2.0 ** -24 * size


def test_another_stream_and_a_graph(ex):
    import torch
    g = torch.Generator().manual_seed(8)
    ptr = _ptr([60, 90]).cuda()
    x = _rand(g, 150, 128, dtype="bfloat16").cuda()
    w, _ = _four(ex, g, 2, 128, 128)
    want = ex.grouped_matmul_mx4(x, w, ptr)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = ex.grouped_matmul_mx4(x, w, ptr, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()

    def all_of_them():
        y = ex.grouped_matmul_mx4(x, w, ptr)
        return y, ex.grouped_matmul_mx4(y, w, ptr, transposed=True), ex.grouped_matmul_mx4(ex.mx4_quantize(y), w, ptr)

    with torch.cuda.graph(graph):
        kept = all_of_them()
    for i in range(4):
        x.copy_(torch.randn(150, 128, device="cuda"))
        ptr.copy_(_ptr([10 * i, 150 - 20 * i]).cuda())
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, all_of_them()):
            assert torch.equal(a, b)


def test_no_groups_and_no_rows(ex):
    import torch
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    x = torch.randn(9, 16, device="cuda")
    none = ex.mx4_quantize(torch.empty(0, 8, 16, device="cuda"))
    assert not ex.grouped_matmul_mx4(x, none, one).any() and not ex.grouped_matmul_mx4(ex.mx4_quantize(x), none, one).any()
    w = ex.mx4_quantize(torch.randn(2, 8, 16, device="cuda"))
    ptr = torch.zeros(3, dtype=torch.int64, device="cuda")
    assert ex.grouped_matmul_mx4(x[:0], w, ptr).shape == (0, 8)
    # numbers of rows of an empty x
    rows = torch.zeros(5, dtype=torch.int32, device="cuda")
    two = torch.tensor([0, 2, 5], device="cuda")
    assert not ex.grouped_matmul_mx4(x[:0], w, two, rows=rows).any() and not ex.grouped_matmul_mx4(ex.mx4_quantize(x[:0]), w, two, rows=rows).any()


def test_refusals(ex):
    import torch
    x = torch.randn(10, 64, device="cuda")
    w = ex.mx4_quantize(torch.randn(2, 8, 64, device="cuda"))
    q = ex.mx4_quantize(x)
    ptr = torch.tensor([0, 4, 10], device="cuda")
    rows = torch.zeros(10, dtype=torch.int32, device="cuda")
    f = ex.grouped_matmul_mx4
    assert f(x, w, ptr).dtype == torch.float32 and f(q, w, ptr).dtype == torch.bfloat16
    for call in (lambda: f(x, w, ptr.int()), lambda: f(x, w, ptr[:2]), lambda: f(x, w, ptr.cpu()), lambda: f(x[:, :63], w, ptr), lambda: f(x, w, ptr, transposed=True),
                 lambda: f(x, w, ptr, rows=rows.long()), lambda: f(x.T, w, ptr), lambda: f(x, w, ptr, out=torch.empty(9, 8, device="cuda")),
                 lambda: f(x, w, ptr, out=torch.empty(10, 8)), lambda: f(x, w, ptr, dtype=torch.float16), lambda: f(x.cpu(), w, ptr), lambda: f(x, q, ptr),
                 lambda: f(q, w, ptr, transposed=True), lambda: f(w, w, ptr), lambda: f(q, w, ptr, dtype=torch.float16, out=torch.empty(10, 8, device="cuda")),
                 lambda: f(ex.mx4_quantize(x[:, :60]), w, ptr)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: f(x.double(), w, ptr), lambda: f(q, w, ptr, dtype=torch.float64)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_sizes_that_take_each_tile(ex, dtype):
    """Of 64 x 64, 128 x 128 and 256 x 256 (16 bits), with lines of whole pieces and without, forward and across, lengths of one step to several and odd ones."""
    for K, N in ((264, 2000), (2000, 264), (1999, 264), (320, 2049), (64, 2560), (2560, 64), (63, 130), (192, 1000), (40, 72)):
        _compare(ex, [1500, 0, 1600], K, N, dtype, K + N, rows_of_x=700)
    _compare(ex, [3000, 3100, 2900, 3300], 2304, 96, dtype, 11)
    _compare(ex, [65, 130, 40], 72, 200, dtype, 12)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_all_rows_in_one_of_many_groups(ex, dtype):
    """Where groups are few rows on the average, one that has them all is shared out in tiles of few rows."""
    _compare(ex, [0] * 7 + [600] + [0] * 60, 200, 136, dtype, 13, rows_of_x=90)
    _compare(ex, [1] * 20 + [150] + [0] * 9 + [17] * 3, 330, 72, dtype, 14)


def test_float16_at_the_ends_of_its_range(ex):
    """Scales at which float16 just holds the matrix's numbers, subnormal ones among them, one step beyond it, zeros at scale 0, and one far scale in a matrix of near ones."""
    import torch
    g = torch.Generator().manual_seed(15)
    for sizes, K, N in (([9], 96, 40), ([200, 130], 96, 150), ([700, 900], 264, 2000)):
        S, E = sum(sizes), len(sizes)
        blocks = (K + 31) // 32
        for low, high in ((104, 112), (103, 106), (138, 140), (140, 142), (90, 150)):
            codes = torch.randint(0, 256, (E, N, blocks * 16), generator=g).to(torch.uint8)
            scales = torch.zeros(E, N, 16, dtype=torch.uint8)
            scales[..., :blocks] = torch.randint(low, high + 1, (E, N, blocks), generator=g).to(torch.uint8)
            codes[:, 3, :16], scales[:, 3, 0] = 0, 0                  # zeros, whatever the scale
            scales[E - 1, N - 1, 1] = 60 if low < 120 else 150          # (beyond float16, in the last tile)
            w, value = ex.Mx4(codes.cuda(), scales.cuda(), K), X.values(X.unpack(codes.numpy()), scales[..., :blocks].numpy().astype(np.int64), K)
            # rows that keep the results within float16
            x = (torch.randn(S, K, generator=g) * (2.0 ** -14 if low >= 120 or high >= 150 else 8.0)).half()
            dy = (torch.randn(S, N, generator=g) * (2.0 ** -14 if low >= 120 or high >= 150 else 8.0)).half()
            ptr = _ptr(sizes)
            want, mag = O.grouped(_np(ptr), _np(x), value)
            with np.errstate(over="ignore"):
                ok = np.abs(want) < 60000
            got = ex.grouped_matmul_mx4(x.cuda(), w, ptr.cuda())
            assert np.all(np.abs(_np(got) - want)[ok] <= (2 * (K + 2) * 2.0 ** -24 * mag + EPS["float16"] * np.abs(want) + TINY["float16"])[ok])
            want, mag = O.grouped(_np(ptr), _np(dy), value.transpose(0, 2, 1))
            ok = np.abs(want) < 60000
            got = ex.grouped_matmul_mx4(dy.cuda(), w, ptr.cuda(), transposed=True)
            assert np.all(np.abs(_np(got) - want)[ok] <= (2 * (N + 2) * 2.0 ** -24 * mag + EPS["float16"] * np.abs(want) + TINY["float16"])[ok])


def test_codes_and_scales_behind_the_end_do_not_count(ex):
    """The same numbers with other bytes behind `inner`, forward, across and with rows in four bits: the same bits."""
    import torch
    g = torch.Generator().manual_seed(16)
    for sizes, K, N in (([3, 9], 70, 50), ([300, 400], 1000, 300), ([40], 4100, 40), ([900], 33, 500)):
        ptr = _ptr(sizes).cuda()
        a = ex.mx4_quantize(torch.randn(len(sizes), N, K, generator=g).cuda())
        q = ex.mx4_quantize(torch.randn(sum(sizes), K, generator=g).cuda())
        x, dy = torch.randn(sum(sizes), K, generator=g).bfloat16().cuda(), torch.randn(sum(sizes), N, generator=g).bfloat16().cuda()

        def other(m):
            codes, scales = m.codes.clone(), m.scales.clone()
            codes[..., (K + 1) // 2:] = 0xff if K % 2 == 0 else codes[..., (K + 1) // 2:]
            if K % 2:
                codes[..., K // 2] |= 0xf0
                codes[..., K // 2 + 1:] = 0x77
            scales[..., (K + 31) // 32:] = 255
            return ex.Mx4(codes, scales, K)

        b, p = other(a), other(q)
        assert torch.equal(ex.grouped_matmul_mx4(x, a, ptr), ex.grouped_matmul_mx4(x, b, ptr))
        assert torch.equal(ex.grouped_matmul_mx4(dy, a, ptr, transposed=True), ex.grouped_matmul_mx4(dy, b, ptr, transposed=True))
        assert torch.equal(ex.grouped_matmul_mx4(q, a, ptr), ex.grouped_matmul_mx4(p, b, ptr))


def test_two_streams_at_once(ex):
    import torch
    g = torch.Generator().manual_seed(17)
    ptr = _ptr([400, 500]).cuda()
    w, _ = _four(ex, g, 2, 300, 520)
    xs = [_rand(g, 900, 520, dtype="bfloat16").cuda() for _ in range(2)]
    want = [(ex.grouped_matmul_mx4(x, w, ptr), ex.grouped_matmul_mx4(ex.mx4_quantize(x), w, ptr)) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for i, (s, x) in enumerate(zip(streams, xs)):
            got[i].append((ex.grouped_matmul_mx4(x, w, ptr, stream=s), ex.grouped_matmul_mx4(ex.mx4_quantize(x, stream=s), w, ptr, stream=s)))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for i in range(2):
        for pair in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(pair, want[i]))
