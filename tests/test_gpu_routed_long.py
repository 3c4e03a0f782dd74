"""The routed products where places in a matrix pass 4 GB: rows beyond the 32-bit range, gathered, written and added up, against 64-bit products
of the rows that are looked at.  Sums of c products in 32 bits are off by (c + 2) * 2^-24 of their magnitudes at most, and are rounded
to bfloat16 once."""
import pytest

from oracle import routed as O

pytestmark = pytest.mark.gpu
LONG, WIDE = 600_000, 4096      # 4.9 GB in bfloat16; element 2^31 is in row 524288


@pytest.fixture(scope="module")
def rt():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import routed
    routed.load()
    return routed


@pytest.fixture(scope="module")
def x():
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randn(LONG, WIDE, device="cuda", dtype=torch.bfloat16, generator=g)


def _rand(seed, *shape):
    import torch
    return torch.randn(*shape, device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(seed))


def _same(got, a, b):
    """got = a b^T, to the roundings."""
    a, b = a.double(), b.double()
    want, mag = a @ b.T, a.abs() @ b.abs().T
    return bool(((got.double() - want).abs() <= (a.shape[1] + 2) * 2.0 ** -24 * mag + 2.0 ** -8 * want.abs() + 2.0 ** -133).all())


@pytest.mark.parametrize("sizes", [[1, 2], [9, 300], [700, 800]])
def test_gathered_rows(rt, x, sizes):
    import torch
    n = sum(sizes)
    rows = torch.randint(0, LONG, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(n), dtype=torch.int32)
    rows[0], rows[-1], rows[n // 2] = LONG - 1, 524288, 524287
    ptr = torch.tensor([0, sizes[0], n], device="cuda")
    w = _rand(2, 2, 72, WIDE)
    kn = w.transpose(1, 2).contiguous()
    dy = _rand(3, n, 72)
    for got in (rt.grouped_matmul(x, w, ptr, rows=rows), rt.grouped_matmul(x, kn, ptr, rows=rows, transposed=True)):
        for e in range(2):
            lo, hi = int(ptr[e]), int(ptr[e + 1])
            assert _same(got[lo:hi], x[rows[lo:hi].long()], w[e])
    dw, dt = rt.grouped_weight_grad(dy, x, ptr, rows=rows), rt.grouped_weight_grad(dy, x, ptr, rows=rows, transposed=True)
    for e in range(2):
        lo, hi = int(ptr[e]), int(ptr[e + 1])
        assert _same(dw[e], dy[lo:hi].T, x[rows[lo:hi].long()].T) and _same(dt[e], x[rows[lo:hi].long()].T, dy[lo:hi].T)


def test_rows_in_order(rt, x):
    import torch
    ptr = torch.tensor([0, 524200, 524300, LONG - 3, LONG], device="cuda")
    w = _rand(4, 4, 24, WIDE)
    got = rt.grouped_matmul(x, w, ptr)
    for e, lo, hi in ((0, 0, 40), (0, 524100, 524200), (1, 524200, 524300), (2, 524300, 524400), (2, LONG - 50, LONG - 3), (3, LONG - 3, LONG)):
        assert _same(got[lo:hi], x[lo:hi], w[e])
    del got
    back = rt.grouped_matmul(_rand(5, LONG, 24), w, ptr, transposed=True)      # the result is long
    dy = _rand(5, LONG, 24)
    for e, lo, hi in ((0, 524100, 524200), (1, 524200, 524300), (3, LONG - 3, LONG)):
        assert _same(back[lo:hi], dy[lo:hi], w[e].T)
    ptr = torch.tensor([524250, 524330, LONG - 90, LONG], device="cuda")
    dw = rt.grouped_weight_grad(dy, x, ptr)
    for e, lo, hi in ((0, 524250, 524330), (2, LONG - 90, LONG)):
        assert _same(dw[e], dy[lo:hi].T, x[lo:hi].T)


def test_adapters(rt, x):
    """(The inner product with A is held in two parts of 16 bits: 2^-15 of the magnitudes at most.)"""
    import torch
    w, a, b = _rand(6, 24, WIDE), _rand(7, 3, 8, WIDE), _rand(8, 3, 24, 8)
    ids = torch.randint(-1, 3, (LONG,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9), dtype=torch.int32)
    y = rt.adapter_matmul(x, w, a, b, ids)
    for lo, hi in ((0, 30), (524270, 524310), (LONG - 30, LONG)):
        want, mag = O.adapter(*(t.double().cpu().numpy() for t in (x[lo:hi], w, a, b)), ids[lo:hi].cpu().numpy())
        got = y[lo:hi].double().cpu().numpy()
        assert (abs(got - want) <= ((WIDE + 12) * 2.0 ** -24 + 2.0 ** -15) * mag + 2.0 ** -8 * abs(want)).all()


def test_combine(rt, x):
    import torch
    T, k = LONG // 2, 2
    logits = torch.randn(T, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(10))
    r = rt.route(logits, k)
    out = rt.combine(x, r)
    dy, dval = rt.combine_backward(out, x, r)
    at = torch.cat([torch.arange(50), torch.arange(T - 50, T)]).cuda()
    slot, val = r.slot.view(T, k)[at].long(), r.val.view(T, k)[at].double()
    assert int(slot.max()) * WIDE > 2 ** 31
    rows = x[slot.view(-1)].view(-1, k, WIDE).double()
    want, mag = (val[:, :, None] * rows).sum(1), (val[:, :, None] * rows).abs().sum(1)
    assert bool(((out[at].double() - want).abs() <= (k + 2) * 2.0 ** -24 * mag + 2.0 ** -8 * want.abs() + 2.0 ** -133).all())
    d = out[at].double()
    wdy = val[:, :, None] * d[:, None, :]
    assert bool(((dy[slot.view(-1)].view(-1, k, WIDE).double() - wdy).abs() <= (2.0 ** -23 + 2.0 ** -8) * wdy.abs() + 2.0 ** -133).all())
    wdval, dmag = (d[:, None, :] * rows).sum(2), (d[:, None, :] * rows).abs().sum(2)
    assert bool(((dval.view(T, k)[at].double() - wdval).abs() <= (WIDE / 32 + 40) * 2.0 ** -24 * dmag).all())


@pytest.mark.parametrize("dtype,inner,more", [("bfloat16", 8, 64), ("bfloat16", 1, 64), ("float32", 1, 3)])
def test_a_row_of_many_columns(rt, dtype, inner, more):
    """More columns than a launch has tiles of 64 x 64 for, whatever the alignment: larger ones are taken."""
    import torch
    t, N = getattr(torch, dtype), (1 << 30) + more
    x = torch.randn(1, inner, device="cuda", generator=torch.Generator(device="cuda").manual_seed(11)).to(t)
    w = torch.empty(1, N, inner, device="cuda", dtype=t)
    for at in range(0, N, 1 << 27):
        w[0, at:at + (1 << 27)].normal_(generator=torch.Generator(device="cuda").manual_seed(at >> 27))
    y = rt.grouped_matmul(x, w, torch.tensor([0, 1], device="cuda"))
    eps = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -24
    for at in range(0, N, 1 << 27):
        a = w[0, at:at + (1 << 27)].double()
        want, mag = (a * x.double()).sum(1), (a * x.double()).abs().sum(1)
        assert bool(((y[0, at:at + (1 << 27)].double() - want).abs() <= (inner + 2) * 2.0 ** -24 * mag + eps * want.abs() + 2.0 ** -133).all()), at


def test_many_rows_of_few_columns(rt):
    import torch
    S, K, N = (1 << 30) + 100, 8, 8
    x = torch.empty(S, K, device="cuda", dtype=torch.bfloat16)
    for at in range(0, S, 1 << 27):
        x[at:at + (1 << 27)].normal_(generator=torch.Generator(device="cuda").manual_seed(at >> 27))
    w = _rand(12, 2, N, K)
    ptr = torch.tensor([5, (1 << 29) + 77, S - 3], device="cuda")
    y = rt.grouped_matmul(x, w, ptr)
    assert not bool(y[:5].any()) and not bool(y[S - 3:].any())
    for lo, hi, e in ((5, 1 << 20, 0), ((1 << 29) - 1000, (1 << 29) + 77, 0), ((1 << 29) + 77, (1 << 29) + 5000, 1), (S - (1 << 20), S - 3, 1)):
        assert _same(y[lo:hi], x[lo:hi], w[e])


def test_adapters_of_many_columns(rt):
    import torch
    M, K, N = 3, 8, (1 << 27) + 24
    x, w, a, b = _rand(13, M, K), _rand(14, N, K), _rand(15, 2, 1, K), _rand(16, 2, N, 1)
    y = rt.adapter_matmul(x, w, a, b, torch.tensor([1, -1, 0], device="cuda", dtype=torch.int32))
    for m, i in ((0, 1), (1, -1), (2, 0)):
        for at in range(0, N, 1 << 25):   # (products and sums: a library's product of a matrix of more than 2^27 rows with a vector is not relied on)
            to = slice(at, at + (1 << 25))
            terms = w[to].double() * x[m].double()
            want, mag = terms.sum(1), terms.abs().sum(1)
            if i >= 0:
                h = a[i, 0].double() * x[m].double()
                want += b[i, to, 0].double() * h.sum()
                mag += b[i, to, 0].double().abs() * h.abs().sum()
            assert bool(((y[m, to].double() - want).abs() <= ((K + 8) * 2.0 ** -24 + 2.0 ** -15) * mag + 2.0 ** -8 * want.abs() + 2.0 ** -133).all()), (m, at)
