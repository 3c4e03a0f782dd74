"""A mixture-of-experts block with adapters in front of it, on the library's routed products: one training step and one decoding step.

    python examples/experts_block.py [tokens] [width] [hidden] [experts] [k]

Training: logits -> routing matrix -> gathered rows through each expert's two matrices -> rows back to their tokens, then the gradients of all
of them, checked against torch.autograd on the same block in single precision.  Decoding: one token for each request, projected
with its request's adapter, through the same block.  At the end the sparse product R^T R: how often two experts are used together.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_19004_amd import binding, routed  # noqa: E402


def silu_grad(h):
    s = torch.sigmoid(h)
    return s * (1 + h * (1 - s))


def forward(x, w_router, w1, w2, k):
    logits = x @ w_router.T
    r = routed.route(logits, k)
    h = routed.grouped_matmul(x, w1, r.expert_ptr, rows=r.token)
    y = routed.grouped_matmul(torch.nn.functional.silu(h), w2, r.expert_ptr)
    return routed.combine(y, r), (logits, r, h, y)


def backward(dout, x, w_router, w1, w2, kept):
    logits, r, h, y = kept
    act = torch.nn.functional.silu(h)
    dy, dval = routed.combine_backward(dout, y, r)
    dact = routed.grouped_matmul(dy, w2, r.expert_ptr, transposed=True)
    dw2 = routed.grouped_weight_grad(dy, act, r.expert_ptr)
    dh = dact * silu_grad(h)
    dw1 = routed.grouped_weight_grad(dh, x, r.expert_ptr, rows=r.token)
    dx = routed.combine(routed.grouped_matmul(dh, w1, r.expert_ptr, transposed=True), r, weighted=False)
    dlogits = routed.route_backward(r, dval, logits)
    return dx + dlogits @ w_router, dlogits.T @ x, dw1, dw2


def with_autograd(x, w_router, w1, w2, k, dout):
    leaves = [t.detach().clone().requires_grad_() for t in (x, w_router, w1, w2)]
    x, w_router, w1, w2 = leaves
    top, col = torch.topk(x @ w_router.T, k, dim=1)
    weight = torch.softmax(top, 1)
    out = torch.zeros_like(dout)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(col == e, as_tuple=True)
        y = torch.nn.functional.silu(x[t] @ w1[e].T) @ w2[e].T
        out = out.index_add(0, t, y * weight[t, j, None])
    out.backward(dout)
    return out.detach(), [t.grad for t in leaves]


def main(tokens=512, width=256, hidden=384, experts=8, k=2):
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std

    x, w_router = normal(tokens, width), normal(experts, width, std=width ** -0.5)
    w1, w2 = normal(experts, hidden, width, std=width ** -0.5), normal(experts, width, hidden, std=hidden ** -0.5)
    dout = normal(tokens, width)
    out, kept = forward(x, w_router, w1, w2, k)
    grads = backward(dout, x, w_router, w1, w2, kept)
    ref, ref_grads = with_autograd(x, w_router, w1, w2, k, dout)
    worst = 0.0
    for name, a, b in zip(("out", "dx", "dw_router", "dw1", "dw2"), (out, *grads), (ref, *ref_grads)):
        worst = max(worst, float((a - b).norm() / b.norm()))
        print(f"training step  {name:10s} off by {float((a - b).norm() / b.norm()):.1e}")

    # decoding: requests with adapters of their own, in 16 bits
    requests, adapters, rank = 24, 6, 16
    low = [t.to(torch.bfloat16) for t in (normal(requests, width), normal(width, width, std=width ** -0.5), normal(adapters, rank, width, std=width ** -0.5),
                                         normal(adapters, width, rank, std=rank ** -0.5))]
    ids = torch.randint(-1, adapters, (requests,), device="cuda", generator=gen, dtype=torch.int32)
    tok = routed.adapter_matmul(*low, ids)
    out, (_, r, _, _) = forward(tok, w_router.to(torch.bfloat16), w1.to(torch.bfloat16), w2.to(torch.bfloat16), k)
    print(f"decoding step  {requests} requests, {int(r.row_ptr[-1])} entries, out {tuple(out.shape)} {out.dtype}")

    # R^T R: R^T in CSR is the routing's own order by experts
    r = kept[1]
    R = r.csr()
    ones = torch.ones_like(R.val)
    C, _ = binding.spgemm(binding.DeviceCSR(experts, tokens, r.expert_ptr, r.token[:R.nnz], ones), binding.DeviceCSR(tokens, experts, R.row_ptr, R.col_idx, ones))
    print(f"used together  {C.nnz} of {experts * experts} pairs of experts, {int(C.val.sum())} times")
    return worst


if __name__ == "__main__":
    sys.exit(0 if main(*(int(a) for a in sys.argv[1:])) < 1e-5 else 1)
