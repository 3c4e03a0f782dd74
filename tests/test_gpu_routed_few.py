"""Products of groups of few rows with long sums, where c is divided among the waves of a workgroup, against 64-bit products on the GPU: rings of stages that are
filled again and end within one, groups of one row to several turns of 64 (32).  Sums of c products in 32 bits are off by (c + 2) * 2^-24
of their magnitudes at most, and are rounded to their type once."""
import pytest

pytestmark = pytest.mark.gpu
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}


@pytest.fixture(scope="module")
def rt():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import routed
    routed.load()
    return routed


def _rand(seed, dtype, *shape):
    import torch
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(getattr(torch, dtype))


def _near(got, want, mag, c, dtype):
    return bool(((got.double() - want).abs() <= (c + 2) * 2.0 ** -24 * mag + EPS[dtype] * want.abs() + TINY[dtype]).all())


def _held(t, off, extra):
    """The same numbers in rows of another stride and base, NaN beside them."""
    import torch
    big = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), device="cuda", dtype=t.dtype)
    big[..., off:off + t.shape[-1]] = t
    return big[..., off:off + t.shape[-1]]


# up to 16 rows, up to 32, up to 64 and several turns, in groups of less than 24 rows on the average
SIZES = [[1, 16, 3], [17, 0, 24, 20], [0, 150, 3, 0, 33, 0, 0, 1], [2, 64, 0, 5, 65, 0, 1, 40]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("c", [768, 1024, 2048, 4096, 4104, 4097])
@pytest.mark.parametrize("n", [72, 456])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_long_sums_of_few_rows(rt, sizes, c, n, dtype):
    import torch
    S, E = sum(sizes), len(sizes)
    assert E * ((n + 63) // 64) < 256 and S <= 24 * E
    x, w = _rand(1, dtype, 50, c), _rand(2, dtype, E, n, c)
    kn = w.transpose(1, 2).contiguous()
    rows = torch.randint(0, 50, (S,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3))
    rows[S // 2] = -1
    ptr = torch.tensor([0] + sizes, device="cuda").cumsum(0)
    left = x.double()[rows.clamp(min=0).long()]
    left[S // 2] = 0
    plain = x[rows.clamp(min=0).long()]
    plain[S // 2] = 0
    calls = {"along": (x, w, rows, False), "across": (x, kn, rows, True), "in order": (plain, w, None, False), "in order, across": (plain, kn, None, True),
             "along, unaligned": (_held(x, 1, 3), _held(w, 3, 5), rows, False), "across, unaligned": (_held(x, 1, 3), _held(kn, 3, 5), rows, True)}
    for name, (x_, w_, rows_, transposed) in calls.items():
        y = rt.grouped_matmul(x_, w_, ptr, rows=rows_, transposed=transposed)
        for e in range(E):
            lo, hi = int(ptr[e]), int(ptr[e + 1])
            a, b = left[lo:hi], w[e].double()
            assert _near(y[lo:hi], a @ b.T, a.abs() @ b.abs().T, c, dtype), (name, e)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("sizes,K,N", [([70, 3, 130], 128, 192), ([9, 0, 14], 136, 72), ([300, 500, 1], 264, 320)])
def test_strides_and_alignment_against_the_definition(rt, sizes, K, N, dtype):
    import torch
    S, ptr = sum(sizes), torch.tensor([0] + sizes, device="cuda").cumsum(0)
    x, w, dy = _rand(1, dtype, S, K), _rand(2, dtype, 3, N, K), _rand(3, dtype, S, N)
    for off, extra in ((0, 0), (8, 64), (1, 3), (4, 12), (0, 1), (2, 66)):
        xs, ws, ds = _held(x, off, extra), _held(w, off, extra), _held(dy, off, extra)
        y, dx = rt.grouped_matmul(xs, ws, ptr), rt.grouped_matmul(ds, ws, ptr, transposed=True)
        held = torch.full((3, N, K + extra), 7.0, device="cuda", dtype=x.dtype)
        dw = rt.grouped_weight_grad(ds, xs, ptr, out=held[:, :, off:off + K])
        dt = rt.grouped_weight_grad(ds, xs, ptr, transposed=True)
        assert bool((held[:, :, :off] == 7).all()) and bool((held[:, :, off + K:] == 7).all())
        for e in range(3):
            lo, hi = int(ptr[e]), int(ptr[e + 1])
            xe, we, de = x[lo:hi].double(), w[e].double(), dy[lo:hi].double()
            for name, got, a, b in (("y", y[lo:hi], xe, we.T), ("dx", dx[lo:hi], de, we), ("dw", dw[e], de.T, xe), ("dt", dt[e], xe.T, de)):
                assert _near(got, a @ b, a.abs() @ b.abs(), a.shape[1], dtype), (name, e, off, extra)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("E,n,c,rows", [(128, 64, 2048, 20), (8, 1024, 4096, 24)])
def test_rows_that_all_meet_in_one_group(rt, E, n, c, rows, transposed):
    """As the routing of a step may have it: right, and no more than four times as long as with the same number in each."""
    import torch
    S = E * rows
    x, w = _rand(1, "bfloat16", S, c), _rand(2, "bfloat16", E, *((c, n) if transposed else (n, c)))
    even, one = torch.arange(E + 1, device="cuda") * rows, torch.zeros(E + 1, device="cuda", dtype=torch.int64)
    one[E // 2 + 1:] = S
    y = rt.grouped_matmul(x, w, one, transposed=transposed)
    a, b = x.double(), w[E // 2].double()
    b = b if transposed else b.T
    assert _near(y, a @ b, a.abs() @ b.abs(), c, "bfloat16")

    def least(ptr):
        times = []
        for _ in range(12):
            s, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            s.record()
            for _ in range(10):
                rt.grouped_matmul(x, w, ptr, transposed=transposed)
            e.record()
            torch.cuda.synchronize()
            times.append(s.elapsed_time(e))
        return min(times)

    least(even)
    assert least(one) <= 4 * least(even)
