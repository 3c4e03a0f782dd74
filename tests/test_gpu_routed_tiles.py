"""Sizes at which each of the tiles is taken (64 x 64 to 256 x 256, straight to LDS and through registers), against 64-bit products on the GPU.
Sums of c products in 32 bits are off by (c + 2) * 2^-24 of their magnitudes at most, and are rounded to their type once."""
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


def _near(got, want, mag, c, dtype, more=0.0):
    return bool(((got.double() - want).abs() <= ((c + 2) * 2.0 ** -24 + more) * mag + EPS[dtype] * want.abs() + TINY[dtype]).all())


def _ptr(sizes):
    import torch
    return torch.tensor([0] + sizes, device="cuda").cumsum(0)


# rows of each group, c, columns: tiles of 256 x 256, 128 x 128, 64 x 128, 64 x 64; the last two through registers (128 x 128, 64 x 64)
ROWS = [([3000, 0, 1192, 4000], 136, 1792), ([3000, 0, 1192, 4000], 136, 2048), ([500, 24, 0, 500], 264, 2176), ([200, 70, 0, 242], 72, 1000),
        ([1500, 1, 1095, 1500], 133, 1001), ([200, 70, 0, 242], 71, 77)]


@pytest.mark.parametrize("sizes,c,n", ROWS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gather", [False, True])
def test_rows(rt, sizes, c, n, dtype, gather):
    import torch
    S = sum(sizes)
    x, w = _rand(1, dtype, 700 if gather else S, c), _rand(2, dtype, len(sizes), n, c)
    rows = torch.randint(-1, 701, (S,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3)) if gather else None
    ptr = _ptr(sizes)
    left = x.double() if rows is None else torch.cat([x, x.new_zeros(2, c)]).double()[torch.where((rows < 0) | (rows > 699), 700, rows).long()]
    held = torch.full((S, n + 3), 7.0, device="cuda", dtype=x.dtype)    # an output whose rows are not whole pieces apart
    for y in (rt.grouped_matmul(x, w, ptr, rows=rows), rt.grouped_matmul(x, w.transpose(1, 2).contiguous(), ptr, rows=rows, transposed=True),
              rt.grouped_matmul(x, w, ptr, rows=rows, out=held[:, 1:n + 1])):
        for e in range(len(sizes)):
            a, b, lo, hi = left[ptr[e]:ptr[e + 1]], w[e].double(), ptr[e], ptr[e + 1]
            assert _near(y[lo:hi], a @ b.T, a.abs() @ b.abs().T, c, dtype), e
    assert bool((held[:, 0] == 7).all()) and bool((held[:, n + 1:] == 7).all())


# outer, inner: tiles of 256 x 256, 128 x 128, 64 x 128, 64 x 64; through registers 128 x 128, 64 x 64
DEPTH = [(2048, 4096), (1024, 2048), (512, 1400), (64, 200), (1001, 1003), (65, 67)]


@pytest.mark.parametrize("outer,inner", DEPTH)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gather", [False, True])
def test_weights(rt, outer, inner, dtype, gather):
    import torch
    sizes = [130, 0, 1, 300]
    S, ptr = sum(sizes), _ptr(sizes)
    x, dy = _rand(1, dtype, 200 if gather else S, inner), _rand(2, dtype, S, outer)
    rows = torch.randint(-1, 201, (S,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3)) if gather else None
    right = x.double() if rows is None else torch.cat([x, x.new_zeros(1, inner)]).double()[torch.where((rows < 0) | (rows > 199), 200, rows).long()]
    dw, dt = rt.grouped_weight_grad(dy, x, ptr, rows=rows), rt.grouped_weight_grad(dy, x, ptr, rows=rows, transposed=True)
    for e in range(4):
        a, b = dy[ptr[e]:ptr[e + 1]].double(), right[ptr[e]:ptr[e + 1]]
        want, mag = a.T @ b, a.abs().T @ b.abs()
        assert _near(dw[e], want, mag, 300, dtype) and _near(dt[e], want.T, mag.T, 300, dtype), e


# rows, c, columns: tiles of 256 x 256, 128 x 256 (single precision: 128 x 128), 64 x 128, 64 x 64; through registers 128 x 128, 64 x 64
ADAPTERS = [(4096, 136, 4096), (6000, 72, 4096), (1200, 264, 2176), (512, 72, 1000), (4096, 133, 1001), (600, 67, 1030)]


@pytest.mark.parametrize("M,c,n", ADAPTERS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("order", ["mixed", "in runs"])
def test_adapters(rt, M, c, n, dtype, order):
    """An inner product with A is held in two parts of 16 bits at least (2^-15 of the magnitudes).  One adapter is broken: its own rows only."""
    import torch
    L, R = 6, 72
    x, w, a, b = _rand(1, dtype, M, c), _rand(2, dtype, n, c), _rand(3, dtype, L, R, c), _rand(4, dtype, L, n, R)
    g = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(-1, L + 1, (M,), device="cuda", dtype=torch.int32, generator=g)
    if order == "in runs":
        ids = ids.sort().values
    ranks, scale = torch.tensor([72, 0, 13, 64, 72, 1], device="cuda", dtype=torch.int32), torch.rand(L, device="cuda", generator=g)
    b[4] = float("nan")
    y = rt.adapter_matmul(x, w, a, b, ids, ranks=ranks, scale=scale)
    want, mag = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    for i in range(L):
        at, r, s = ids == i, int(ranks[i]), float(scale[i])
        h, hm = x[at].double() @ a[i, :r].double().T, x[at].double().abs() @ a[i, :r].double().abs().T
        want[at] += s * h @ b[i, :, :r].double().T
        mag[at] += s * hm @ b[i, :, :r].double().abs().T
    broken = ids == 4
    assert bool(y[broken].isnan().all())
    floor = 2.0 ** -25 * 512 if dtype == "float16" else 0.0
    assert bool(((y.double() - want).abs() <= ((c + R + 4) * 2.0 ** -24 + (0.0 if dtype == "float32" else 2.0 ** -15)) * mag + EPS[dtype] * want.abs() + TINY[dtype]
                 + floor)[~broken].all())


@pytest.mark.parametrize("outer,inner", DEPTH)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_slots_whose_row_is_outside_add_nothing(rt, outer, inner, dtype):
    """Whatever their gradient holds, as their product is 0 whatever the matrix holds."""
    import torch
    sizes = [130, 0, 1, 300]
    S, ptr = sum(sizes), _ptr(sizes)
    x, dy = _rand(1, dtype, 200, inner), _rand(2, dtype, S, outer)
    rows = torch.randint(0, 200, (S,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(3))
    out = torch.arange(S, device="cuda") % 5 == 2
    rows[out] = torch.tensor([-1, 200, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int32).repeat(S)[:int(out.sum())]
    dy[out] = float("nan")
    dy[::10][out[::10]] = float("inf")
    right = torch.where(out[:, None], 0.0, x.double()[rows.clamp(0, 199).long()])
    left = torch.where(out[:, None], 0.0, dy.double())
    dw, dt = rt.grouped_weight_grad(dy, x, ptr, rows=rows), rt.grouped_weight_grad(dy, x, ptr, rows=rows, transposed=True)
    for e in range(4):
        a, b = left[ptr[e]:ptr[e + 1]], right[ptr[e]:ptr[e + 1]]
        want, mag = a.T @ b, a.abs().T @ b.abs()
        assert _near(dw[e], want, mag, 300, dtype) and _near(dt[e], want.T, mag.T, 300, dtype), e
    w = _rand(4, dtype, 4, outer, inner)
    w[:, 0, 0] = float("inf")
    assert not bool(rt.grouped_matmul(x, w, ptr, rows=rows)[out].any())
    assert not bool(rt.grouped_matmul(x, w.transpose(1, 2).contiguous(), ptr, rows=rows, transposed=True)[out].any())
