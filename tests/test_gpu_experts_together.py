"""A router's losses, its experts in four bits and the routed products together, as a training step and a decoding step use them, against autograd in 64 bits, eagerly
and captured."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts, routed
    experts.load()
    return routed, experts


def _step(lib, x, w_router, w1, w2, k, dout, dloss):
    """Loss and gradients of rows and router of a block whose experts are frozen in four bits."""
    import torch
    rt, ex = lib
    logits = x @ w_router.T
    r = rt.route(logits, k)
    b = ex.route_balance(logits, r)
    h = ex.grouped_matmul_mx4(x, w1, r.expert_ptr, rows=r.token)
    act = torch.relu(h)
    y = ex.grouped_matmul_mx4(act, w2, r.expert_ptr)
    out = rt.combine(y, r)
    dy, dval = rt.combine_backward(dout, y, r)
    dh = ex.grouped_matmul_mx4(dy, w2, r.expert_ptr, transposed=True) * (h > 0)
    dx = rt.combine(ex.grouped_matmul_mx4(dh, w1, r.expert_ptr, transposed=True), r, weighted=False)
    dlogits = ex.route_balance_backward(b, r, logits, dloss, dval=dval)
    return out, b.loss, dx + dlogits @ w_router, dlogits.T @ x


def _in_64_bits(lib, x, w_router, w1, w2, k, dout, dloss):
    import torch
    _, ex = lib
    x, w_router = (t.detach().double().requires_grad_() for t in (x, w_router))
    w1, w2 = (ex.mx4_dequantize(w, torch.float32).double() for w in (w1, w2))
    logits = x @ w_router.T
    E = logits.shape[1]
    top, col = torch.topk(logits, k, dim=1)
    weight = torch.softmax(top, 1)
    out = torch.zeros_like(dout, dtype=torch.float64)
    for e in range(E):
        t, j = torch.nonzero(col == e, as_tuple=True)
        out = out.index_add(0, t, torch.relu(x[t] @ w1[e].T) @ w2[e].T * weight[t, j, None])
    share = torch.bincount(col.reshape(-1), minlength=E).double() / col.numel()
    loss = torch.stack([E * (share * torch.softmax(logits, 1).mean(0)).sum(), (torch.logsumexp(logits, 1) ** 2).mean()])
    ((out * dout).sum() + (loss * dloss).sum()).backward()
    return out.detach(), loss.detach(), x.grad, w_router.grad


def _inputs(ex, T, D, F, E, seed):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=g) * std

    w1, w2 = ex.mx4_quantize(normal(E, F, D, std=D ** -0.5)), ex.mx4_quantize(normal(E, D, F, std=F ** -0.5))
    return normal(T, D), normal(E, D, std=D ** -0.5), w1, w2, normal(T, D), torch.tensor([3.0, 0.5], device="cuda")


@pytest.mark.parametrize("T,D,F,E,k", [(1, 64, 96, 4, 2), (40, 72, 40, 5, 3), (600, 256, 320, 16, 4)])
def test_a_training_step_around_frozen_experts(lib, T, D, F, E, k):
    x, w_router, w1, w2, dout, dloss = _inputs(lib[1], T, D, F, E, T + D)
    got = _step(lib, x, w_router, w1, w2, k, dout, dloss)
    want = _in_64_bits(lib, x, w_router, w1, w2, k, dout, dloss)
    # single precision: four products in a row, each off by about sqrt(c) * 2^-24 of its norm or less, the softmax' some ten roundings: 1e-5 is tenfold
    for a, b in zip(got, want):
        assert float((a.double() - b).norm() / b.norm()) < 1e-5


def test_captured_beside_eager_steps(lib):
    import torch
    x, w_router, w1, w2, dout, dloss = _inputs(lib[1], 200, 128, 160, 8, 7)
    w_router = w_router.clone()
    for _ in range(2):
        _step(lib, x, w_router, w1, w2, 2, dout, dloss)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = _step(lib, x, w_router, w1, w2, 2, dout, dloss)
    for i in range(4):
        x.copy_(torch.randn(200, 128, device="cuda"))
        dloss.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, _step(lib, x, w_router, w1, w2, 2, dout, dloss)):
            assert torch.allclose(a, b, rtol=1e-5, atol=1e-5 * float(b.abs().max()))   # (a library's products beside the library's own)


@pytest.mark.parametrize("requests", [1, 24])
def test_a_decoding_step_in_four_bits(lib, requests):
    """bfloat16 rows, then rows in four bits: against the same numbers in 64 bits, each product rounded to bfloat16."""
    import torch
    rt, ex = lib
    x, w_router, w1, w2, _, _ = _inputs(ex, requests, 256, 384, 8, requests)
    x = x.bfloat16()
    d1, d2 = (ex.mx4_dequantize(w, torch.float32).double() for w in (w1, w2))
    r = rt.route((x.float() @ w_router.T), 2)
    for four in (False, True):
        rows = ex.mx4_quantize(x) if four else x
        h = torch.relu(ex.grouped_matmul_mx4(rows, w1, r.expert_ptr, rows=r.token))
        y = ex.grouped_matmul_mx4(ex.mx4_quantize(h) if four else h, w2, r.expert_ptr)
        assert h.dtype == y.dtype == torch.bfloat16
        xd, hd = (ex.mx4_dequantize(ex.mx4_quantize(t), torch.float32).double() if four else t.double() for t in (x, h))
        ptr = r.expert_ptr.tolist()
        for e in range(8):
            at = slice(ptr[e], ptr[e + 1])
            for got, a, b, least in ((h[at], xd[r.token[at].long()], d1[e], 0.0), (y[at], hd[at], d2[e], float("-inf"))):
                want, mag = (a @ b.T).clamp(min=least), a.abs() @ b.abs().T
                within = (got.double() - want).abs() <= 386 * 2.0 ** -24 * mag + 2.0 ** -8 * want.abs()
                assert int((~within).sum()) == 0
