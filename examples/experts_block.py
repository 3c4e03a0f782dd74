"""A mixture-of-experts block with adapters in front of it, on the library's routed products: one training step and one decoding step.

    python examples/experts_block.py [tokens] [width] [hidden] [experts] [k]

Training: logits -> routing matrix and the losses that keep the experts evenly used -> gathered rows through each expert's two matrices -> rows back to
their tokens, then the gradients of all of them, checked against torch.autograd on the same block in single precision.  Decoding: one token for each request,
projected with its request's adapter, through the same block, then through the experts in four bits, checked against the same numbers in single
precision.  At the end the sparse product R^T R: how often two experts are used together.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_19004_amd import binding, experts, routed  # noqa: E402


def silu_grad(h):
    s = torch.sigmoid(h)
    return s * (1 + h * (1 - s))


def forward(x, w_router, w1, w2, k):
    logits = x @ w_router.T
    r = routed.route(logits, k)
    h = routed.grouped_matmul(x, w1, r.expert_ptr, rows=r.token)
    y = routed.grouped_matmul(torch.nn.functional.silu(h), w2, r.expert_ptr)
    return routed.combine(y, r), (logits, r, h, y)


def forward_in_four_bits(x, w_router, w1, w2, k):
    r = routed.route(x @ w_router.T, k)
    h = experts.grouped_matmul_mx4(experts.mx4_quantize(x), w1, r.expert_ptr, rows=r.token)
    y = experts.grouped_matmul_mx4(experts.mx4_quantize(torch.nn.functional.silu(h)), w2, r.expert_ptr)
    return routed.combine(y, r), (r, h)


def backward(dout, dloss, x, w_router, w1, w2, kept, balance):
    logits, r, h, y = kept
    act = torch.nn.functional.silu(h)
    dy, dval = routed.combine_backward(dout, y, r)
    dact = routed.grouped_matmul(dy, w2, r.expert_ptr, transposed=True)
    dw2 = routed.grouped_weight_grad(dy, act, r.expert_ptr)
    dh = dact * silu_grad(h)
    dw1 = routed.grouped_weight_grad(dh, x, r.expert_ptr, rows=r.token)
    dx = routed.combine(routed.grouped_matmul(dh, w1, r.expert_ptr, transposed=True), r, weighted=False)
    dlogits = experts.route_balance_backward(balance, r, logits, dloss, dval=dval)
    return dx + dlogits @ w_router, dlogits.T @ x, dw1, dw2


def with_autograd(x, w_router, w1, w2, k, dout, dloss):
    leaves = [t.detach().clone().requires_grad_() for t in (x, w_router, w1, w2)]
    x, w_router, w1, w2 = leaves
    logits = x @ w_router.T
    top, col = torch.topk(logits, k, dim=1)
    weight = torch.softmax(top, 1)
    out = torch.zeros_like(dout)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(col == e, as_tuple=True)
        y = torch.nn.functional.silu(x[t] @ w1[e].T) @ w2[e].T
        out = out.index_add(0, t, y * weight[t, j, None])
    E = w1.shape[0]
    share = torch.bincount(col.reshape(-1), minlength=E) / col.numel()
    loss = torch.stack([E * (share * torch.softmax(logits, 1).mean(0)).sum(), (torch.logsumexp(logits, 1) ** 2).mean()])
    ((out * dout).sum() + (loss * dloss).sum()).backward()
    return out.detach(), loss.detach(), [t.grad for t in leaves]


def main(tokens=512, width=256, hidden=384, count=8, k=2):
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, device="cuda", generator=gen) * std

    x, w_router = normal(tokens, width), normal(count, width, std=width ** -0.5)
    w1, w2 = normal(count, hidden, width, std=width ** -0.5), normal(count, width, hidden, std=hidden ** -0.5)
    dout, dloss = normal(tokens, width), torch.tensor([10.0, 1.0], device="cuda")
    out, kept = forward(x, w_router, w1, w2, k)
    balance = experts.route_balance(kept[0], kept[1])
    grads = backward(dout, dloss, x, w_router, w1, w2, kept, balance)
    ref, ref_loss, ref_grads = with_autograd(x, w_router, w1, w2, k, dout, dloss)
    worst = 0.0
    for name, a, b in zip(("out", "losses", "dx", "dw_router", "dw1", "dw2"), (out, balance.loss, *grads), (ref, ref_loss, *ref_grads)):
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

    # the same requests through the experts in four bits; what the first product gives before its rounding to 16 bits, from the numbers that the codes stand for
    four = [experts.mx4_quantize(t) for t in (w1, w2)]
    out, (r, h) = forward_in_four_bits(tok, w_router.to(torch.bfloat16), *four, k)
    rows, w = experts.mx4_dequantize(experts.mx4_quantize(tok), torch.float32), experts.mx4_dequantize(four[0], torch.float32)
    expert = torch.repeat_interleave(torch.arange(count, device="cuda"), r.expert_ptr.diff().long())
    ref = torch.stack([w[e] @ rows[t] for e, t in zip(expert.tolist(), r.token.tolist())])
    off = float(((h.float() - ref).abs() / (2 ** -8 * ref.abs() + 1e-5 * ref.abs().max())).max())
    print(f"in four bits   out {tuple(out.shape)} {out.dtype}, the first product within {off:.2f} of a rounding to 16 bits")
    worst = max(worst, 0.0 if off <= 1.0 else off)

    # R^T R: R^T in CSR is the routing's own order by experts
    r = kept[1]
    R = r.csr()
    ones = torch.ones_like(R.val)
    C, _ = binding.spgemm(binding.DeviceCSR(count, tokens, r.expert_ptr, r.token[:R.nnz], ones), binding.DeviceCSR(tokens, count, R.row_ptr, R.col_idx, ones))
    print(f"used together  {C.nnz} of {count * count} pairs of experts, {int(C.val.sum())} times")
    return worst


if __name__ == "__main__":
    sys.exit(0 if main(*(int(a) for a in sys.argv[1:])) < 1e-5 else 1)
