"""Matrices in microscaled four bits (mx4_quantize, mx4_dequantize): codes and scales are equal to those of the definition, and what is read back to the numbers."""
import numpy as np
import pytest

from oracle import experts as X

pytestmark = pytest.mark.gpu
DTYPES = ["float32", "bfloat16", "float16"]


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts
    experts.load()
    return experts


def _np(t):
    return t.detach().cpu().double().numpy()


def _same(ex, x, q):
    """q is x's quantisation, and reads back as that."""
    import torch
    flat = _np(x).reshape(-1, x.shape[-1])
    codes, scales = X.quantize(flat)
    blocks = scales.shape[1]
    got = X.unpack(q.codes.cpu().numpy()).reshape(codes.shape)
    have = q.scales.cpu().numpy().reshape(len(flat), -1)
    assert np.array_equal(have[:, :blocks], scales)
    bad = np.repeat(scales == 255, 32, axis=1)
    # (a negative zero may keep its sign or not)
    assert np.array_equal(np.where(bad, 0, got) & np.where(got % 8, 15, 7), np.where(bad, 0, codes) & np.where(codes % 8, 15, 7))
    want = torch.from_numpy(X.values(codes, scales, x.shape[-1]).reshape(x.shape))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        assert torch.equal(ex.mx4_dequantize(q, dtype).cpu().nan_to_num(nan=12345.0), want.to(dtype).nan_to_num(nan=12345.0)), dtype


@pytest.mark.parametrize("shape", [(1, 1), (1, 32), (3, 31), (5, 33), (2, 128), (7, 200), (4, 3, 96), (2, 9, 1001), (3, 2048), (1, 8193), (300, 64)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_codes_and_scales(ex, shape, dtype):
    import torch
    g = torch.Generator().manual_seed(sum(shape))
    x = (torch.randn(*shape, generator=g) * torch.exp(torch.randn(*shape[:-1], 1, generator=g) * 3)).to(getattr(torch, dtype))
    _same(ex, x, ex.mx4_quantize(x.cuda()))


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_limits_and_zeros(ex, dtype):
    """Numbers at and next to each border between codes, at scales from the smallest to the largest that the type has, subnormal ones too."""
    import torch
    t = getattr(torch, dtype)
    info = torch.finfo(t)
    v = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0], dtype=torch.float64)
    low, high = (-26, 12) if dtype == "float16" else (-151, 125)
    rows = []
    for e in sorted(set(list(range(low, low + 12)) + [-20, -3, 0, 1, 5, 9] + list(range(high - 3, high + 1)))):
        for eps in (0.0, 2.0 ** -7, -2.0 ** -7):
            part = v * (1 + eps) * 2.0 ** e
            rows.append(torch.cat([part, -part]))
    x = torch.stack(rows).to(t)
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, info.max))
    x = torch.cat([x, torch.zeros(2, 32, dtype=t), torch.full((1, 32), info.max, dtype=t), torch.full((1, 32), -info.max, dtype=t), torch.full((1, 32), info.tiny, dtype=t)])
    x[-5, 3] = -0.0
    _same(ex, x, ex.mx4_quantize(x.cuda()))


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_numbers_and_nan_make_their_block_nan(ex, dtype):
    import torch
    x = torch.randn(6, 100).to(getattr(torch, dtype))
    x[0, 5], x[1, 99], x[2, 40], x[3, 64] = float("inf"), float("nan"), float("-inf"), float("nan")
    q = ex.mx4_quantize(x.cuda())
    _same(ex, x, q)
    back = ex.mx4_dequantize(q, torch.float32).cpu()
    assert back[0, :32].isnan().all() and not back[0, 32:].isnan().any() and back[1, 96:].isnan().all() and not back[4:].isnan().any()


def test_every_code_at_every_scale_is_read_back(ex):
    import torch
    codes = torch.arange(256).to(torch.uint8).repeat(256, 1)[:, :16 * 16]
    scales = torch.arange(256).to(torch.uint8)[:, None].repeat(1, 16)
    q = ex.Mx4(codes.cuda(), scales.cuda(), 512)
    want = torch.from_numpy(X.values(X.unpack(codes.numpy()), scales.numpy().astype(np.int64), 512))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        w = want.to(torch.float32).to(dtype)   # (of numbers beyond float16: rounded once, as every number here is one of single precision, or infinite there)
        assert torch.equal(ex.mx4_dequantize(q, dtype).cpu().nan_to_num(nan=12345.0), w.nan_to_num(nan=12345.0)), dtype


def test_strides_and_what_lies_beside(ex):
    import torch
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        x = torch.randn(3, 10, 77).to(dtype).cuda()
        want = ex.mx4_quantize(x)
        for off, extra in ((0, 3), (1, 4), (8, 24)):
            held = torch.full((3, 10, 77 + extra + off), float("nan"), dtype=dtype, device="cuda")
            held[..., off:off + 77] = x
            codes = torch.full((3, 12, 16 * 5), 9, dtype=torch.uint8, device="cuda")
            scales = torch.full((3, 11, 48), 9, dtype=torch.uint8, device="cuda")
            q = ex.mx4_quantize(held[..., off:off + 77], out=ex.Mx4(codes[:, 1:11, 16:64], scales[:, 1:, 16:32], 77))
            assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
            codes[:, 1:11, 16:64] = 9
            scales[:, 1:, 16:32] = 9
            assert bool((codes == 9).all()) and bool((scales == 9).all())
            out = torch.full((3, 10, 77 + extra + off), 7.0, dtype=dtype, device="cuda")
            ex.mx4_dequantize(want, out=out[..., off:off + 77])
            assert torch.equal(out[..., off:off + 77], ex.mx4_dequantize(want, dtype))
            assert bool((out[..., :off] == 7).all()) and bool((out[..., off + 77:] == 7).all())


def test_codes_behind_the_end_do_not_count(ex):
    import torch
    x = torch.randn(4, 40).cuda()
    q = ex.mx4_quantize(x)
    assert not q.codes[:, 20:].any() and not q.scales[:, 2:].any()
    q.codes[:, 20:], q.scales[:, 2:] = 0xff, 0xff
    _same(ex, x.cpu(), ex.Mx4(q.codes.index_fill(1, torch.arange(20, 32, device="cuda"), 0), q.scales, 40))
    assert torch.equal(ex.mx4_dequantize(q, torch.float32), ex.mx4_dequantize(ex.mx4_quantize(x), torch.float32))


def test_empty_ones_streams_and_graphs(ex):
    import torch
    for shape in ((0, 5), (5, 0), (0, 3, 4), (3, 0, 4)):
        q = ex.mx4_quantize(torch.empty(shape, device="cuda"))
        assert q.shape == shape and ex.mx4_dequantize(q).shape == shape
    x = torch.randn(70, 96, device="cuda").to(torch.bfloat16)
    want = ex.mx4_quantize(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = ex.mx4_quantize(x, stream=s)
    back = ex.mx4_dequantize(q, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(q.codes, want.codes) and torch.equal(back, ex.mx4_dequantize(want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = ex.mx4_quantize(x)
        back = ex.mx4_dequantize(q, torch.float32)
    for i in range(3):
        x.copy_(torch.randn(70, 96, device="cuda") * 10 ** i)
        graph.replay()
        torch.cuda.synchronize()
        want = ex.mx4_quantize(x)
        assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales) and torch.equal(back, ex.mx4_dequantize(want, torch.float32))


def test_more_rows_than_a_launch_has_threads_for(ex):
    """Short rows beyond the grid's limit are gone through in turns."""
    import torch
    n = (1 << 26) + 5
    x = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")
    x[::1000003] = 3.0
    x[-1] = -5.5
    back = ex.mx4_dequantize(ex.mx4_quantize(x))
    x[-1] = -6.0   # (5.5 is between 4 and 6, nearer to 6)
    assert torch.equal(back, x)


def test_laid_out_copies_what_does_not_lie_as_wanted(ex):
    import copy
    import torch
    x = torch.randn(3, 8, 90).cuda()
    q = ex.mx4_quantize(x)
    back = ex.mx4_dequantize(q, torch.float32)
    odd = torch.empty(3, 8, 16 * 3 + 1, dtype=torch.uint8, device="cuda")[..., 1:]
    odd.copy_(q.codes)
    p = ex.Mx4.laid_out(odd, q.scales[..., :3].contiguous(), 90)
    assert torch.equal(ex.mx4_dequantize(p, torch.float32), back)
    p = ex.Mx4.laid_out(q.codes.transpose(0, 1).contiguous().transpose(0, 1), q.scales[..., :3], 90)
    assert torch.equal(ex.mx4_dequantize(p, torch.float32), back)
    c = copy.deepcopy(q)
    assert c.codes.data_ptr() != q.codes.data_ptr() and torch.equal(ex.mx4_dequantize(c, torch.float32), back)
    assert torch.equal(ex.mx4_dequantize(ex.Mx4(q.codes[1:], q.scales[1:], 90), torch.float32), back[1:])


def test_refusals(ex):
    import torch
    x = torch.randn(6, 64, device="cuda")
    q = ex.mx4_quantize(x)
    for call in (lambda: ex.mx4_quantize(x.T), lambda: ex.mx4_quantize(x[0]), lambda: ex.mx4_quantize(x[:5], out=q), lambda: ex.mx4_quantize(x.cpu()),
                 lambda: ex.mx4_dequantize(q, out=torch.empty(6, 63, device="cuda")), lambda: ex.mx4_dequantize(q, torch.float16, out=torch.empty(6, 64, device="cuda")),
                 lambda: ex.mx4_dequantize(q, out=torch.empty(6, 64)),
                 lambda: ex.mx4_quantize(x.expand(2, 6, 64), out=ex.Mx4(q.codes.expand(2, 6, 32), q.scales.expand(2, 6, 16), 64))):
        with pytest.raises((ValueError, RuntimeError)):
            call()
    with pytest.raises(TypeError):
        ex.mx4_quantize(x.double())
    with pytest.raises(TypeError):
        ex.mx4_dequantize(q, torch.float64)
