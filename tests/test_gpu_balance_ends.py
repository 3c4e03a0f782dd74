"""The losses of a router through the C ABI with what they read and nothing else, and where their sums are large."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2604_19004_amd import experts
    experts.load()
    return experts


def test_a_routing_of_what_is_read(ex):
    """tokens, experts and expert_ptr for the losses, tokens and experts for their gradient: the bits of the whole routing's."""
    import torch
    from paper_2604_19004_amd import routed
    lib, s = ex.load(), torch.cuda.current_stream().cuda_stream
    x = torch.randn(300, 21, device="cuda")
    r, g = routed.route(x, 3), torch.tensor([0.7, 0.2], device="cuda")
    b = ex.route_balance(x, r)
    d = ex.route_balance_backward(b, r, x, g)
    bare = ex.ocean_routing(300, 21, 0, 0, None, None, None, r.expert_ptr.data_ptr(), None, None)
    nbytes = lib.ocean_route_balance_workspace(300, 21)
    space = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    c = ex.Balance(*(torch.zeros_like(t) for t in (b.loss, b.counts, b.prob, b.rows)))
    out = torch.zeros_like(x)
    held = ex.ocean_balance(c.loss.data_ptr(), c.counts.data_ptr(), c.prob.data_ptr(), c.rows.data_ptr())
    assert lib.ocean_route_balance(ctypes.byref(bare), x.data_ptr(), 1, 21, ctypes.byref(held), space.data_ptr(), nbytes, s) == 0
    bare.expert_ptr = None
    assert lib.ocean_route_balance_backward(ctypes.byref(held), ctypes.byref(bare), x.data_ptr(), 1, 21, g.data_ptr(), None, 1, out.data_ptr(), 21, s) == 0
    assert torch.equal(c.loss, b.loss) and torch.equal(c.counts, b.counts) and torch.equal(c.prob, b.prob) and torch.equal(c.rows, b.rows) and torch.equal(out, d)


@pytest.mark.parametrize("E", [1, 5, 100, 700])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_squares_whose_sum_is_beyond_single_precision(ex, E, dtype):
    """Logits about 1.5e19: the mean of logsumexp^2, 2.25e38, is a number of single precision, the sum of two of them is not.  A row's logsumexp is its largest logit (the others are
    further below than exp reaches) or that plus log of how often it is there, which single precision does not tell from it, so the mean is one of exact squares, rounded once; 300
    additions in 64 bits, or 32, add at most as many roundings."""
    import torch
    from paper_2604_19004_amd import routed
    gen = torch.Generator().manual_seed(E)
    x = (torch.rand(300, E, generator=gen) * 0.6e19 + 1.2e19).to(getattr(torch, dtype))
    x[7] = float("-inf")
    d = x.cuda()
    b = ex.route_balance(d, routed.route(d, 1))
    top = np.delete(x.double().amax(1).numpy(), 7)
    want = float((top ** 2).mean())
    assert 1.4e38 < want < 3.3e38 and float((top ** 2).sum()) > 1e40
    assert int(b.rows) == 299 and abs(float(b.loss[1]) - want) <= 302 * 2.0 ** -24 * want
