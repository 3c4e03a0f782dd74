"""A shared projection with adapters of many requests (adapter_matmul) against its definition in 64 bits.

Tolerance: sums of c products in 32 bits are off by at most (c + 1) * 2^-24 of the sum of their magnitudes.  In the adapter's part every
magnitude passes through two such sums (inner, then rank), the scale and, for 16-bit types, the halving of the inner product in two
parts of 16 bits (bfloat16: 2 * 2^-8 * 2^-8 = 2^-16 at most).  Then one rounding to the type."""
import numpy as np
import pytest

from oracle import routed as O

pytestmark = pytest.mark.gpu
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}   # half a unit in the last place, relative
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}
HALVES = {"float32": 0.0, "bfloat16": 2.0 ** -15, "float16": 2.0 ** -15}


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
    # (float16: what is left of a small inner product may be a subnormal number, 2^-25 off, times up to some hundred numbers of about 4)
    floor = 2.0 ** -25 * 512 if dtype == "float16" else 0.0
    return bool(np.all(np.abs(_np(got) - want) <= ((c + 4) * 2.0 ** -24 + HALVES[dtype]) * mag + EPS[dtype] * np.abs(want) + TINY[dtype] + floor))


def _case(M, K, N, R, L, dtype, seed, plain=0.2):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = getattr(torch, dtype)
    x, w = torch.randn(M, K, generator=g).to(t), torch.randn(N, K, generator=g).to(t)
    a, b = torch.randn(L, R, K, generator=g).to(t), (torch.randn(L, N, R, generator=g) * 0.2).to(t)
    ids = torch.randint(0, max(L, 1), (M,), generator=g, dtype=torch.int32)
    ids[torch.rand(M, generator=g) < plain] = -1
    return x, w, a, b, ids


# one row to several tiles; ranks below, at and beyond a piece, a step and a tile; odd sizes
CASES = [(1, 64, 64, 8, 1), (1, 8, 8, 1, 1), (3, 1, 1, 1, 2), (48, 256, 128, 16, 64), (64, 200, 72, 13, 9), (65, 128, 136, 64, 3), (130, 67, 33, 24, 5),
         (301, 200, 101, 24, 9), (300, 320, 520, 33, 4), (520, 136, 264, 128, 7), (290, 72, 264, 256, 2), (700, 128, 256, 16, 40), (5, 0, 16, 8, 2),
         (5, 16, 24, 0, 2), (5, 16, 24, 8, 0), (17, 4096, 40, 16, 20)]


@pytest.mark.parametrize("M,K,N,R,L", CASES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("ragged", [False, True])
def test_against_the_definition(rt, M, K, N, R, L, dtype, ragged):
    import torch
    x, w, a, b, ids = _case(M, K, N, R, L, dtype, M + K + N + R + L)
    g = torch.Generator().manual_seed(1)
    ranks = torch.randint(0, R + 1, (L,), generator=g, dtype=torch.int32) if ragged else None
    scale = torch.rand(L, generator=g) * 2 if ragged else None
    want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids), None if ranks is None else _np(ranks), None if scale is None else _np(scale))
    if ragged:   # what lies behind an adapter's rank is not used
        for i in range(L):
            a[i, ranks[i]:] = float("nan")
            b[i, :, ranks[i]:] = float("inf")
    got = rt.adapter_matmul(x.cuda(), w.cuda(), a.cuda(), b.cuda(), ids.cuda(), ranks=None if ranks is None else ranks.cuda(),
                            scale=None if scale is None else scale.cuda())
    assert got.shape == (M, N) and _close(got, want, mag, K + R, dtype)


@pytest.mark.parametrize("M", [9, 200, 600])
def test_a_broken_adapter_harms_its_own_rows_only(rt, M):
    import torch
    x, w, a, b, ids = _case(M, 128, 264, 16, 5, "bfloat16", 3)
    want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids))
    for bad in (float("nan"), float("inf")):
        a2, b2, w2 = a.clone(), b.clone(), w
        a2[1], b2[2] = bad, bad
        got = rt.adapter_matmul(x.cuda(), w2.cuda(), a2.cuda(), b2.cuda(), ids.cuda())
        ok = (ids != 1) & (ids != 2)
        assert _close(got[ok.cuda()], want[ok.numpy()], mag[ok.numpy()], 144, "bfloat16")
        assert not bool(torch.isfinite(got[(~ok).cuda()]).any())


@pytest.mark.parametrize("M", [40, 500])
def test_ids_outside_the_table_and_ranks_outside_their_range(rt, M):
    import torch
    x, w, a, b, ids = _case(M, 64, 64, 8, 4, "float16", 4)
    ids[::3] = torch.tensor([4, 100, -7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).repeat(M)[:len(ids[::3])]
    ranks = torch.tensor([-3, 0, 50, 8], dtype=torch.int32)
    want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids), np.array([0, 0, 8, 8]))
    assert _close(rt.adapter_matmul(x.cuda(), w.cuda(), a.cuda(), b.cuda(), ids.cuda(), ranks=ranks.cuda()), want, mag, 72, "float16")


@pytest.mark.parametrize("M", [30, 300])
def test_strides_and_alignment(rt, M):
    import torch
    K, N, R, L = 128, 264, 16, 6
    x, w, a, b, ids = (t.cuda() for t in _case(M, K, N, R, L, "bfloat16", 5))
    want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids))

    def held(t, off, extra):
        big = torch.full((*t.shape[:-1], t.shape[-1] + extra), float("nan"), device="cuda", dtype=t.dtype)
        big[..., off:off + t.shape[-1]] = t
        return big[..., off:off + t.shape[-1]]

    for off, extra in ((8, 16), (1, 3), (4, 4), (2, 6)):
        out = torch.full((M, N + extra), 7.0, device="cuda", dtype=x.dtype)
        rt.adapter_matmul(held(x, off, extra), held(w, off, extra), held(a, off, extra), held(b, off, extra), ids, out=out[:, off:off + N])
        assert _close(out[:, off:off + N], want, mag, K + R, "bfloat16")
        assert bool((out[:, :off] == 7).all()) and bool((out[:, off + N:] == 7).all())


def test_the_same_result_each_time_on_any_stream_and_from_a_graph(rt):
    import torch
    for M in (33, 900):
        x, w, a, b, ids = (t.cuda() for t in _case(M, 512, 256, 32, 12, "bfloat16", 6))
        want = rt.adapter_matmul(x, w, a, b, ids)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        y = rt.adapter_matmul(x, w, a, b, ids, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = rt.adapter_matmul(x, w, a, b, ids)
        for i in range(4):
            ids.copy_(torch.randint(-1, 12, (M,), dtype=torch.int32))
            x.copy_(torch.randn(M, 512))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, rt.adapter_matmul(x, w, a, b, ids))


def test_refusals(rt):
    import ctypes
    import torch
    x, w, a, b, ids = (t.cuda() for t in _case(10, 32, 24, 8, 3, "bfloat16", 7))
    for call in (lambda: rt.adapter_matmul(x, w[:, :16], a, b, ids), lambda: rt.adapter_matmul(x, w, a[:, :4], b, ids), lambda: rt.adapter_matmul(x, w, a, b[:2], ids),
                 lambda: rt.adapter_matmul(x, w, a, b, ids[:9]), lambda: rt.adapter_matmul(x, w, a, b, ids.long()), lambda: rt.adapter_matmul(x, w.half(), a, b, ids),
                 lambda: rt.adapter_matmul(x, w, a.cpu(), b, ids), lambda: rt.adapter_matmul(x, w, a, b, ids, ranks=ids), lambda: rt.adapter_matmul(x, w, a, b, ids, scale=torch.ones(3)),
                 lambda: rt.adapter_matmul(x, w, a[0], b, ids), lambda: rt.adapter_matmul(x, w, a, b, ids, out=x),
                 lambda: rt.adapter_matmul(x, w, torch.empty(1, 257, 32, device="cuda", dtype=x.dtype), torch.empty(1, 24, 257, device="cuda", dtype=x.dtype), ids)):
        with pytest.raises(ValueError):
            call()
    lib = rt.load()
    y = torch.empty(10, 24, device="cuda", dtype=x.dtype)
    need = lib.ocean_adapter_workspace(10, 32, 24, 3, 8, 2)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(dtype=2, ids_=ids.data_ptr(), ld_x=32, bytes_=need, rank=8, adapters=3, ldb=8):
        c = rt.ocean_adapters(adapters, rank, a.data_ptr(), 32, 256, b.data_ptr(), ldb, 192, None, None)
        return lib.ocean_adapter_matmul(ctypes.byref(c), ids_, dtype, 10, 32, 24, x.data_ptr(), ld_x, w.data_ptr(), 32, y.data_ptr(), 24, space.data_ptr(), bytes_, None)

    assert call() == 0
    for rc, word in ((lambda: call(dtype=0), "dtype"), (lambda: call(ids_=None), "ids"), (lambda: call(ld_x=31), "stride"), (lambda: call(bytes_=need - 1), "workspace"),
                     (lambda: call(rank=257), "rank"), (lambda: call(adapters=-1), "range"), (lambda: call(ldb=7), "stride")):
        assert rc() == 1 and word in lib.ocean_last_error().decode()
    assert lib.ocean_adapter_workspace(10, 32, 24, 3, 300, 2) == 0


def _same_with_infinities(got, want, bound):
    """NaN where the definition has one, its infinities, and finite results to the bound."""
    g = _np(got)
    finite = np.isfinite(want)
    return bool(np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(g[np.isinf(want)], want[np.isinf(want)])
                and np.all(np.abs(g[finite] - want[finite]) <= bound[finite]))


@pytest.mark.parametrize("M", [9, 1200])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_infinite_inner_products_and_matrices(rt, M, dtype):
    """An infinity follows the definition, however many rows there are: adapter 0 has one infinite inner product, adapter 1 also one of some hundred
    thousand (beyond float16) the other way, adapters 2 and 3 an infinite number of B beside inner products of either size and of no remainder."""
    import torch
    K, N, R, L = 64, 264, 20, 5
    x, w, a, b, _ = _case(M, K, N, R, L, dtype, 11)
    x = x.abs().clamp(min=0.5, max=2)
    b[b == 0] = 1
    ids = torch.arange(M, dtype=torch.int32) % (L + 1) - 1
    a[0, 3] = float("inf")
    a[1, 3], a[1, 4], b[1, :, 3], b[1, :, 4] = float("inf"), 4096, 0.5, -0.25
    a[2] = a[2].abs() + 0.5
    b[2, 5, 0], b[2, 200, 19], b[2, 7, 8] = float("inf"), float("-inf"), float("nan")
    a[3] = 0
    a[3, :, 0], x[:, 0], b[3, 9, 2] = 0.25, 0.5, float("inf")     # inner products of 1 / 8: nothing is left of them
    with np.errstate(invalid="ignore"):
        want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids))
    rows = [[m for m in range(M) if ids[m] == i] for i in range(L)]
    assert np.isinf(want[rows[0]]).all() and (want[rows[1]] == np.inf).all() and np.isinf(want[rows[2]][:, [5, 200]]).all() and (want[rows[3]][:, 9] == np.inf).all()
    bound = ((K + R + 4) * 2.0 ** -24 + HALVES[dtype]) * np.nan_to_num(mag, nan=0, posinf=0) + EPS[dtype] * np.abs(np.nan_to_num(want, posinf=0, neginf=0)) + TINY[dtype]
    got = rt.adapter_matmul(x.cuda(), w.cuda(), a.cuda(), b.cuda(), ids.cuda())
    assert _same_with_infinities(got, want, bound)


@pytest.mark.parametrize("M", [9, 2500])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("ratio", [20, 26, 28])
def test_small_inner_products_beside_large_ones(rt, M, dtype, ratio):
    """A row's inner products are 2^13 and 2^(13 - ratio), and B takes the small one only.  Of the largest 2^-39 may be lost (float16), of each 2^-15."""
    import torch
    K, N, R = 64, 136, 9
    t = getattr(torch, dtype)
    x, w = torch.ones(M, K).to(t), torch.zeros(N, K).to(t)
    a, b = torch.zeros(1, R, K), torch.zeros(1, N, R)
    a[0, 2, 0], a[0, 7, 1:3], b[0, :, 7] = 2.0 ** 13, 2.0 ** (12 - ratio) * 1.25, 8.0
    b[0, ::3, 7] = -16.0
    a, b = a.to(t), b.to(t)
    assert float(a[0, 7, 1]) == 2.0 ** (12 - ratio) * 1.25
    ids = torch.zeros(M, dtype=torch.int32)
    want, mag = O.adapter(_np(x), _np(w), _np(a), _np(b), _np(ids))
    got = _np(rt.adapter_matmul(x.cuda(), w.cuda(), a.cuda(), b.cuda(), ids.cuda()))
    lost = 2.0 ** -39 * 2.0 ** 13 * 16 if dtype == "float16" else 0.0
    assert np.all(np.abs(got - want) <= ((K + R + 4) * 2.0 ** -24 + HALVES[dtype]) * mag + EPS[dtype] * np.abs(want) + TINY[dtype] + lost)
    assert np.all(np.abs(want) > 8 * lost)
