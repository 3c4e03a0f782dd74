"""Products with rows in four bits that lie far apart (gathered from more than 4 GB, or with long strides), and rows just below the 4 GB that 32-bit offsets reach."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts
    experts.load()
    yield experts
    torch.cuda.empty_cache()


def _numbers(ex, q):
    import torch
    return ex.mx4_dequantize(q, torch.float32)


def _near(got, x, w, c):
    """got against x @ w.T in 64 bits: (c + 2) roundings of the magnitudes and one to the type."""
    import torch
    x, w = x.double(), w.double()
    want, mag = x @ w.T, x.abs() @ w.abs().T
    return bool(((got.double() - want).abs() <= (c + 2) * 2.0 ** -24 * mag + torch.finfo(got.dtype).eps / 2 * want.abs()).all())


def _codes(gen, *shape):
    import torch
    return torch.randint(0, 256, shape, device="cuda", generator=gen, dtype=torch.uint8)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_many_rows_gathered_from_far(ex, dtype):
    """More slots than go 16 at a time (2^20), from 4.4 GB of codes, in lines that end inside a block: the first and last of each group, both ends of x, and others."""
    import torch
    g = torch.Generator("cuda").manual_seed(1)
    n, K, N, S = 1 << 21, 4224 - 5, 40, (1 << 20) + 5000
    w = ex.mx4_quantize(torch.randn(2, N, K, device="cuda", generator=g))
    x = ex.Mx4(_codes(g, n, 2112), torch.randint(122, 132, (n, 144), device="cuda", generator=g, dtype=torch.uint8), K)
    rows = torch.randint(0, n, (S,), device="cuda", generator=g, dtype=torch.int32)
    rows[0], rows[1], rows[S - 1], rows[S - 2] = n - 1, 0, n - 2, n // 2
    rows[70], rows[S - 70] = -1, n
    middle = S // 3 + 1
    y = ex.grouped_matmul_mx4(x, w, torch.tensor([0, middle, S], device="cuda"), rows=rows, dtype=getattr(torch, dtype))
    assert not y[70].any() and not y[S - 70].any()
    for e, (lo, hi) in enumerate(((0, middle), (middle, S))):
        at = torch.cat([torch.arange(lo, lo + 200), torch.randint(lo, hi, (2000,)), torch.arange(hi - 200, hi)]).cuda()
        at = at[(rows[at] >= 0) & (rows[at] < n)]
        near = rows[at].long()
        assert _near(y[at], _numbers(ex, ex.Mx4(x.codes[near], x.scales[near], K)), _numbers(ex, w)[e], K)


@pytest.mark.parametrize("sizes,N,K", [([100, 200], 70, 500), ([40, 260], 1100, 512), ([13, 287], 33, 31), ([290, 10], 130, 2048 + 64)])
def test_rows_with_long_strides(ex, sizes, N, K):
    """Rows 2^24 bytes and more apart, of codes or of scales, gathered or not: as those of a copy that lies close together."""
    import torch
    g = torch.Generator("cuda").manual_seed(2)
    S, blocks = sum(sizes), (K + 31) // 32
    width, up = 16 * blocks, (blocks + 15) // 16 * 16
    w = ex.mx4_quantize(torch.randn(2, N, K, device="cuda", generator=g))
    ptr = torch.tensor([0, sizes[0], S], device="cuda")
    wd = _numbers(ex, w)
    rows = torch.randperm(S, device="cuda", generator=g).to(torch.int32)
    far = torch.zeros(S, (1 << 24) + 48, device="cuda", dtype=torch.uint8)
    for held in ("codes", "scales"):
        codes, scales = _codes(g, S, width), torch.randint(120, 130, (S, up), device="cuda", generator=g, dtype=torch.uint8)
        if held == "codes":
            far[:, 32:32 + width] = codes
            x = ex.Mx4(far[:, 32:32 + width], scales, K)
        else:
            far[:, 48:48 + up] = scales
            x = ex.Mx4(codes, far[:, 48:48 + up], K)
        xd = _numbers(ex, ex.Mx4(codes, scales, K))
        for dtype in (torch.float32, torch.bfloat16):
            for index in (None, rows):
                y = ex.grouped_matmul_mx4(x, w, ptr, rows=index, dtype=dtype)
                xs = xd if index is None else xd[index.long()]
                assert _near(y[:sizes[0]], xs[:sizes[0]], wd[0], K) and _near(y[sizes[0]:], xs[sizes[0]:], wd[1], K), (held, dtype, index is None)


@pytest.mark.parametrize("four", [False, True])
def test_rows_just_within_reach(ex, four):
    """x just below the 4 GB (less 64 KB) that 32-bit offsets are taken for, straight to LDS: its last rows and those about 2 GB, where the offsets' highest bit begins."""
    import torch
    g = torch.Generator("cuda").manual_seed(3)
    K = 4224 if four else 1056
    n = ((1 << 32) - 65536 - 1) // 2112
    w = ex.mx4_quantize(torch.randn(2, 300, K, device="cuda", generator=g))
    wd = _numbers(ex, w)
    if four:
        x = ex.Mx4(_codes(g, n, 2112), torch.full((n, 144), 127, device="cuda", dtype=torch.uint8), K)
    else:
        x = torch.empty(n, K, device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    assert (1 << 32) - 65536 - 2112 <= n * 2112 < (1 << 32) - 65536
    for S in (150, 1500, 9000):
        rows = torch.randint(0, n, (S,), device="cuda", generator=g, dtype=torch.int32)
        half = (1 << 31) // 2112
        rows[:6] = torch.tensor([n - 1, n - 2, 0, half - 1, half, half + 1], dtype=torch.int32)
        rows[S - 2:] = torch.tensor([n - 1, half], dtype=torch.int32)
        ptr = torch.tensor([0, S // 3, S], device="cuda")
        y = ex.grouped_matmul_mx4(x, w, ptr, rows=rows, **({"dtype": torch.bfloat16} if four else {}))
        at = rows.long()
        xd = _numbers(ex, ex.Mx4(x.codes[at], x.scales[at], K)) if four else x[at]
        assert _near(y[:S // 3], xd[:S // 3], wd[0], K) and _near(y[S // 3:], xd[S // 3:], wd[1], K), S
