"""Products in which every row chooses its matrix: what they are measured on, their plain forms, and what they should give.

A routing matrix (tokens x experts, a few entries a row) is a sparse matrix in CSR.  Four operators belong to it:

  route     the matrix from logits, its entries in the order of the experts, and the gradient of the logits
  combine   the matrix times the dense rows that the experts gave (one row an entry), and its two gradients
  grouped   the products of ragged groups of rows with their expert's weights: forward, with the weights stored either way,
            and backward (gradient of the rows, gradient of the weights)
  adapter   a shared projection with a low-rank adapter for each row beside it, adapters of many requests in one batch

Inputs are resident in device memory.  A program that serves or trains a mixture of experts holds the routing of a batch
while it makes the products, one that serves adapters holds every adapter in one padded table.
"""
import math
import zlib

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the router of one decoding step: a batch of requests, one token each; latency is all there is
        {"name": "route-decode", "op": "route", "tokens": 64, "experts": 64, "k": 4, "dtype": "bf16", "normalize": True,
         "pad": 0, "closed": 0, "backward": False},
        # a training step's router, forward and backward: probabilities over all experts, some experts closed, padded tokens
        {"name": "route-train", "op": "route", "tokens": 32768, "experts": 100, "k": 8, "dtype": "f32", "normalize": False,
         "pad": 500, "closed": 4, "backward": True},
        # the end of an experts' block for an odd batch of single tokens
        {"name": "combine-decode", "op": "combine", "tokens": 37, "experts": 16, "k": 2, "width": 2047, "dtype": "f16",
         "pad": 0, "weighted": True, "backward": False},
        # the same in training, both gradients, with padded tokens
        {"name": "combine-train", "op": "combine", "tokens": 16384, "experts": 64, "k": 4, "width": 2048, "dtype": "bf16",
         "pad": 300, "weighted": True, "backward": True},
        # one token through two of eight experts: the bytes of two weight matrices
        {"name": "grouped-token", "op": "grouped", "tokens": 1, "experts": 8, "k": 2, "inner": 4096, "outer": 8192, "dtype": "bf16",
         "layout": "nk", "pad": 0, "closed": 0, "backward": False},
        # a decoding batch over many small experts: ragged groups of none to a few dozen rows
        {"name": "grouped-batch", "op": "grouped", "tokens": 96, "experts": 64, "k": 6, "inner": 2048, "outer": 1536, "dtype": "f16",
         "layout": "nk", "pad": 0, "closed": 2, "backward": False},
        # a prompt through eight experts: thousands of rows each, the matrix cores' case
        {"name": "grouped-prompt", "op": "grouped", "tokens": 16384, "experts": 8, "k": 2, "inner": 4096, "outer": 8192,
         "dtype": "bf16", "layout": "nk", "pad": 100, "closed": 0, "backward": False},
        # a training step's backward pass: gradients of the rows and of the weights, an odd number of rows in every group
        {"name": "grouped-train", "op": "grouped", "tokens": 8192, "experts": 32, "k": 4, "inner": 2048, "outer": 1400, "dtype": "bf16",
         "layout": "nk", "pad": 33, "closed": 1, "backward": True},
        # the same in single precision at sizes that no vector load divides, weights stored the other way
        {"name": "grouped-odd-f32", "op": "grouped", "tokens": 777, "experts": 5, "k": 2, "inner": 1001, "outer": 515, "dtype": "f32",
         "layout": "kn", "pad": 7, "closed": 0, "backward": True},
        # a decoding step of requests that each have an adapter of their own
        {"name": "adapter-decode", "op": "adapter", "rows": 48, "inner": 4096, "outer": 4096, "rank": 16, "adapters": 64,
         "requests": 48, "dtype": "bf16", "plain_rows": 0.1, "ragged": False},
        # packed prompts of a few requests
        {"name": "adapter-prompt", "op": "adapter", "rows": 6000, "inner": 4096, "outer": 4096, "rank": 64, "adapters": 32,
         "requests": 12, "dtype": "bf16", "plain_rows": 0.1, "ragged": False},
        # adapters of different ranks, short prompts and single tokens together, sizes that no tile divides
        {"name": "adapter-odd", "op": "adapter", "rows": 301, "inner": 2000, "outer": 1001, "rank": 24, "adapters": 9,
         "requests": 40, "dtype": "f16", "plain_rows": 0.2, "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: half of them multiples of 64, a quarter multiples of 8, the others as they fall."""
    n = _log_int(rng, lo, hi)
    step = rng.choice([64, 64, 8, 1])
    n = max(step, n // step * step)
    return n - step if n == 3072 else n


def draw(rng):
    op = rng.choice(["route", "combine", "grouped", "grouped", "grouped", "adapter", "adapter"])
    if op == "route":
        experts = _log_int(rng, 2, 512)
        k = min(experts, rng.randint(1, 8))
        tokens = min(_log_int(rng, 1, 65536), 6000000 // experts)
        return {"op": op, "tokens": tokens, "experts": experts, "k": k, "dtype": rng.choice(["bf16", "f16", "f32"]),
                "normalize": rng.random() < 0.5, "pad": rng.choice([0, tokens // 20]),
                "closed": rng.choice([0, experts // 10]), "backward": rng.random() < 0.5}
    if op == "combine":
        experts, width = _log_int(rng, 2, 128), _width(rng, 64, 8192)
        k = min(experts, rng.randint(1, 8))
        tokens = max(1, min(_log_int(rng, 1, 32768), 100000000 // (k * width)))
        return {"op": op, "tokens": tokens, "experts": experts, "k": k, "width": width, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "pad": rng.choice([0, tokens // 20]), "weighted": rng.random() < 0.75, "backward": rng.random() < 0.5}
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
    inner, outer = _width(rng, 128, 8192), _width(rng, 128, 8192)
    most = (1 << 40) if dtype != "f32" else (1 << 38)   # products
    if op == "grouped":
        experts = max(1, min(_log_int(rng, 2, 128), (200000000 if dtype != "f32" else 60000000) // (inner * outer)))
        k = min(experts, rng.randint(1, 8))
        backward = rng.random() < 0.4
        tokens = max(1, min(_log_int(rng, 1, 16384), most // (4 if backward else 2) // (k * inner * outer), (1 << 27) // (k * (inner + outer))))
        return {"op": op, "tokens": tokens, "experts": experts, "k": k, "inner": inner, "outer": outer, "dtype": dtype,
                "layout": rng.choice(["nk", "nk", "kn"]), "pad": rng.choice([0, tokens // 20]), "closed": rng.choice([0, (experts - k) // 4]),
                "backward": backward}
    rows = max(1, min(_log_int(rng, 1, 8192), most // 2 // (inner * outer)))
    return {"op": op, "rows": rows, "inner": inner, "outer": outer, "rank": rng.choice([4, 8, 16, 16, 24, 32, 64, 128, 13]),
            "adapters": _log_int(rng, 1, 128), "requests": rng.randint(1, min(rows, 200)), "dtype": dtype,
            "plain_rows": rng.choice([0.0, 0.1, 0.3]), "ragged": rng.random() < 0.3}


# ----------------------------------------------------------------- inputs
def _case_generator(case):
    shape = sorted((k, v) for k, v in case.items() if k != "name")
    return torch.Generator(device=DEVICE).manual_seed(zlib.crc32(repr(shape).encode()))


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed * 7919 + 13)


def _normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, device=DEVICE, generator=gen) * std).to(dtype)


def _routing(case, seed):
    """A routing of case's tokens: k experts a token, some experts in more demand than others, the last `pad` tokens and the
    first `closed` experts with nothing.  It is drawn once per case; the seed turns the numbering of the tokens that take part."""
    T, E, k = case["tokens"], case["experts"], case["k"]
    live = T - case["pad"]
    gen = _case_generator(case)
    demand = torch.randn(E, device=DEVICE, generator=gen) * 0.7
    score = demand - torch.log(-torch.log(torch.rand(live, E, device=DEVICE, generator=gen).clamp(1e-9, 1 - 1e-7)))
    score[:, :case.get("closed", 0)] = -math.inf
    chosen = torch.sort(torch.topk(score, k, dim=1).indices, dim=1).values
    chosen = torch.roll(chosen, seed * 2654435761 % 1000003 % max(live, 1), 0)
    flat = chosen.reshape(-1)
    row_ptr = torch.arange(T + 1, device=DEVICE).clamp(max=live) * k
    expert_ptr = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE)
    torch.cumsum(torch.bincount(flat, minlength=E), 0, out=expert_ptr[1:])
    col_idx, token, slot = (torch.full((T * k,), -1, dtype=torch.int32, device=DEVICE) for _ in range(3))
    order = torch.sort(flat, stable=True).indices
    col_idx[:flat.numel()] = flat.to(torch.int32)
    token[:flat.numel()] = (order // k).to(torch.int32)
    slot[order] = torch.arange(flat.numel(), dtype=torch.int32, device=DEVICE)
    return {"row_ptr": row_ptr, "col_idx": col_idx, "expert_ptr": expert_ptr, "token": token, "slot": slot}


def _inputs(case, seed):
    gen, dtype, op = _generator(seed), TYPES[case["dtype"]], case["op"]
    d = {}
    if op == "route":
        T, E = case["tokens"], case["experts"]
        d["logits"] = _normal(gen, T, E, std=1.5, dtype=dtype)
        d["logits"][:, :case["closed"]] = -math.inf
        d["logits"][T - case["pad"]:] = torch.finfo(dtype).min
        if case["backward"]:
            d["dval"] = _normal(gen, T * case["k"])
    elif op == "combine":
        d.update(_routing(case, seed))
        T, k, D = case["tokens"], case["k"], case["width"]
        val = torch.rand(T, k, device=DEVICE, generator=gen) + 0.05
        d["val"] = (val / val.sum(1, keepdim=True)).reshape(-1) if case["weighted"] else None
        d["y"] = _normal(gen, T * k, D, dtype=dtype)
        if case["backward"]:
            d["dout"] = _normal(gen, T, D, dtype=dtype)
    elif op == "grouped":
        d.update(_routing(case, seed))
        T, E, K, N = case["tokens"], case["experts"], case["inner"], case["outer"]
        d["x"] = _normal(gen, T, K, dtype=dtype)
        shape = (E, N, K) if case["layout"] == "nk" else (E, K, N)
        d["w"] = _normal(gen, *shape, std=K ** -0.5, dtype=dtype)
        if case["backward"]:
            d["dy"] = _normal(gen, T * case["k"], N, dtype=dtype)
    else:
        M, K, N, R, L = case["rows"], case["inner"], case["outer"], case["rank"], case["adapters"]
        plan = _case_generator(case)
        cuts = torch.randperm(max(M - 1, 1), device=DEVICE, generator=plan)[:case["requests"] - 1] + 1 if M > 1 else torch.zeros(0, device=DEVICE)
        request = torch.zeros(M + 1, dtype=torch.int64, device=DEVICE)
        request[cuts.long()] = 1
        request = torch.cumsum(request[:M], 0)
        of_request = torch.randint(0, L, (case["requests"],), device=DEVICE, generator=plan)
        plain = torch.rand(case["requests"], device=DEVICE, generator=plan) < case["plain_rows"]
        of_request = torch.where(plain, -1, of_request)
        d["ids"] = torch.roll(of_request[request], seed * 2654435761 % 1000003 % M, 0).to(torch.int32)
        d["ranks"] = torch.randint(1, R + 1, (L,), device=DEVICE, generator=plan).to(torch.int32) if case["ragged"] else None
        d["scale"] = torch.rand(L, device=DEVICE, generator=gen) + 0.5
        d["x"] = _normal(gen, M, K, dtype=dtype)
        d["w"] = _normal(gen, N, K, std=K ** -0.5, dtype=dtype)
        d["a"] = _normal(gen, L, R, K, std=K ** -0.5, dtype=dtype)
        d["b"] = _normal(gen, L, N, R, std=R ** -0.5, dtype=dtype)
    return d


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2604_19004_amd import routed
        if case["op"] == "combine":
            state["routing"] = routed.Routing(case["tokens"], case["experts"], case["k"], state["row_ptr"], state["col_idx"], state["val"],
                                              state["expert_ptr"], state["token"], state["slot"])
    elif case["op"] == "grouped":
        state["sizes"] = (state["expert_ptr"][1:] - state["expert_ptr"][:-1]).tolist()
    elif case["op"] == "adapter":
        ids = state["ids"].tolist()
        state["used"] = [(a, torch.tensor([i for i, x in enumerate(ids) if x == a], device=DEVICE)) for a in sorted(set(ids) - {-1})]
    return state


# ------------------------------------------------------------ plain forms
def _plain_route(case, logits, dval):
    T, E, k, dtype = case["tokens"], case["experts"], case["k"], logits.dtype
    x = logits.float()
    limits = torch.finfo(dtype)
    x = torch.where(torch.isnan(x) | (x <= limits.min), -math.inf, x.clamp(max=limits.max))
    column = torch.arange(E, device=DEVICE)
    left, cols, vals = x, [], []
    for _ in range(k):
        top = left.amax(1, keepdim=True)
        col = torch.where((left == top) & (top > -math.inf), column, E).amin(1, keepdim=True)
        cols.append(col)
        vals.append(top)
        left = torch.where(column == col, -math.inf, left)
    cols, order = torch.sort(torch.cat(cols, 1), dim=1)
    vals = torch.cat(vals, 1).gather(1, order)
    found = cols < E
    top = vals.amax(1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    e = torch.exp(vals - top)
    every = None
    if case["normalize"]:
        total = e.sum(1, keepdim=True)
    else:
        every = torch.exp(x - top)
        total = every.sum(1, keepdim=True)
    total = torch.where(total > 0, total, 1.0)
    weight = e / total

    row_ptr = torch.zeros(T + 1, dtype=torch.int64, device=DEVICE)
    torch.cumsum(found.sum(1), 0, out=row_ptr[1:])
    place = torch.where(found, row_ptr[:-1, None] + torch.arange(k, device=DEVICE), T * k)   # (entries that are not there: behind the end)
    col_idx = torch.full((T * k + 1,), -1, dtype=torch.int64, device=DEVICE)
    val = torch.zeros(T * k + 1, device=DEVICE)
    row = torch.full((T * k + 1,), -1, dtype=torch.int64, device=DEVICE)
    col_idx.scatter_(0, place.reshape(-1), torch.where(found, cols, -1).reshape(-1))
    val.scatter_(0, place.reshape(-1), torch.where(found, weight, 0.0).reshape(-1))
    row.scatter_(0, place.reshape(-1), torch.where(found, torch.arange(T, device=DEVICE)[:, None], -1).reshape(-1))
    col_idx, val, row = col_idx[:-1], val[:-1], row[:-1]
    key, entry = torch.sort(torch.where(col_idx < 0, E, col_idx), stable=True)
    expert_ptr = (key[None, :] < torch.arange(E + 1, device=DEVICE)[:, None]).sum(1) if E * T * k <= 1 << 22 else \
        torch.searchsorted(key, torch.arange(E + 1, device=DEVICE))
    slot = torch.zeros_like(entry)
    slot[entry] = torch.arange(T * k, device=DEVICE)
    slot = torch.where(col_idx < 0, -1, slot)
    out = {"row_ptr": row_ptr, "col_idx": col_idx.to(torch.int32), "val": val, "expert_ptr": expert_ptr,
           "token": row[entry].to(torch.int32), "slot": slot.to(torch.int32)}
    if dval is not None:
        g = torch.where(found, dval[place.clamp(max=T * k - 1)], 0.0)
        weight = torch.where(found, weight, 0.0)
        mean = (weight * g).sum(1, keepdim=True)
        sparse = weight * g if every is not None else weight * (g - mean)
        grad = torch.zeros(T, E + 1, device=DEVICE).scatter_add_(1, torch.where(found, cols, E), sparse)[:, :E]
        if every is not None:
            grad = grad - every / total * mean
        out["dlogits"] = grad.to(dtype)
    return out


def _entries_by_row(case, row_ptr):
    at = row_ptr[:-1, None] + torch.arange(case["k"], device=DEVICE)
    there = at < row_ptr[1:, None]
    return torch.where(there, at, 0), there


def _plain_combine(case, s):
    at, there = _entries_by_row(case, s["row_ptr"])
    slot = torch.where(there, s["slot"][at].long(), 0)
    y = s["y"].float()
    weight = torch.where(there, s["val"][at] if s["val"] is not None else 1.0, 0.0)
    if not case["backward"]:
        return (y[slot] * weight[:, :, None]).sum(1).to(s["y"].dtype)
    dout = s["dout"].float()
    dy = torch.zeros_like(y)
    dval = torch.zeros(at.numel(), device=DEVICE)
    first = case["tokens"] - case["pad"]   # (padded tokens come last and have no entries)
    for j in range(case["k"]):
        dy[slot[:first, j]] = dout[:first] * weight[:first, j, None]
        dval[at[:first, j]] = (dout[:first] * y[slot[:first, j]]).sum(1)
    return {"dy": dy.to(s["y"].dtype), "dval": dval}


def _plain_grouped(case, s):
    x, w, rows = s["x"].float(), s["w"].float(), s["token"].long()
    if case["layout"] == "kn":
        w = w.transpose(1, 2)
    ends = [0]
    for n in s["sizes"]:
        ends.append(ends[-1] + n)
    slots, dtype = rows.numel(), s["x"].dtype
    if not case["backward"]:
        y = torch.zeros(slots, case["outer"], device=DEVICE)
        for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
            if hi > lo:
                y[lo:hi] = x[rows[lo:hi]] @ w[e].T
        return y.to(dtype)
    dy = s["dy"].float()
    dx = torch.zeros(slots, case["inner"], device=DEVICE)
    dw = torch.zeros(s["w"].shape, device=DEVICE)
    for e, (lo, hi) in enumerate(zip(ends, ends[1:])):
        if hi > lo:
            dx[lo:hi] = dy[lo:hi] @ w[e]
            xe = x[rows[lo:hi]]
            dw[e] = dy[lo:hi].T @ xe if case["layout"] == "nk" else xe.T @ dy[lo:hi]
    return {"dx": dx.to(dtype), "dw": dw.to(dtype)}


def _plain_adapter(case, s):
    x, a, b = s["x"].float(), s["a"], s["b"]
    y = x @ s["w"].float().T
    ids, R = s["ids"].long(), case["rank"]
    has = ids >= 0
    safe = ids.clamp(min=0)
    scale = torch.where(has, s["scale"][safe], 0.0)
    rank = s["ranks"][safe] if s["ranks"] is not None else torch.full_like(safe, R)
    live = torch.arange(R, device=DEVICE) < rank[:, None]
    if case["rows"] * R * max(case["inner"], case["outer"]) <= 1 << 27:
        h = (x[:, None, :] * a[safe].float()).sum(2) * live
        y = y + scale[:, None] * (b[safe].float() * h[:, None, :]).sum(2)
    else:
        for i, at in s["used"]:
            h = (x[at] @ a[i].float().T) * live[at]
            y[at] = y[at] + scale[at, None] * (h @ b[i].float().T)
    return y.to(s["x"].dtype)


# -------------------------------------------------------------------- run
def run(state):
    case, op = state["case"], state["case"]["op"]
    if not own:
        if op == "route":
            return _plain_route(case, state["logits"], state.get("dval"))
        return {"combine": _plain_combine, "grouped": _plain_grouped, "adapter": _plain_adapter}[op](case, state)
    from paper_2604_19004_amd import routed
    if op == "route":
        r = routed.route(state["logits"], case["k"], normalize=case["normalize"])
        out = {"row_ptr": r.row_ptr, "col_idx": r.col_idx, "val": r.val, "expert_ptr": r.expert_ptr, "token": r.token, "slot": r.slot}
        if case["backward"]:
            out["dlogits"] = routed.route_backward(r, state["dval"], state["logits"], normalize=case["normalize"])
        return out
    if op == "combine":
        if not case["backward"]:
            return routed.combine(state["y"], state["routing"])
        dy, dval = routed.combine_backward(state["dout"], state["y"], state["routing"])
        return {"dy": dy, "dval": dval}
    if op == "grouped":
        kn = case["layout"] == "kn"
        if not case["backward"]:
            return routed.grouped_matmul(state["x"], state["w"], state["expert_ptr"], rows=state["token"], transposed=kn)
        dx = routed.grouped_matmul(state["dy"], state["w"], state["expert_ptr"], transposed=not kn)
        dw = routed.grouped_weight_grad(state["dy"], state["x"], state["expert_ptr"], rows=state["token"], transposed=kn)
        return {"dx": dx, "dw": dw}
    return routed.adapter_matmul(state["x"], state["w"], state["a"], state["b"], state["ids"], ranks=state["ranks"], scale=state["scale"])


# ------------------------------------------------- what it should come to
def _exact_route(case, d):
    logits, T, E, k = d["logits"], case["tokens"], case["experts"], case["k"]
    info = torch.finfo(logits.dtype)
    open_ = (logits > info.min)          # (neither NaN nor -inf is)
    x = torch.where(open_, logits.double().clamp(max=float(info.max)), -math.inf)
    best, col = torch.sort(x, dim=1, descending=True, stable=True)
    take = torch.zeros(T, E, dtype=torch.bool, device=DEVICE).scatter_(1, col[:, :k], best[:, :k] > -math.inf)
    counts = take.sum(1)
    t, e = torch.nonzero(take, as_tuple=True)
    some = open_.any(1)
    p = torch.zeros(T, E, dtype=torch.float64, device=DEVICE)
    p[some] = torch.softmax((torch.where(take, x, -math.inf) if case["normalize"] else x)[some], dim=1)
    n, cap = t.numel(), T * k

    def filled(values, fill, dtype):
        out = torch.full((cap,), fill, dtype=dtype, device=DEVICE)
        out[:n] = values.to(dtype)
        return out

    row_ptr = torch.zeros(T + 1, dtype=torch.int64, device=DEVICE)
    row_ptr[1:] = torch.cumsum(counts, 0)
    by_expert = torch.nonzero(take.T.contiguous())
    number = torch.zeros(T, E, dtype=torch.int64, device=DEVICE)
    number[by_expert[:, 1], by_expert[:, 0]] = torch.arange(n, device=DEVICE)
    expert_ptr = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE)
    expert_ptr[1:] = torch.cumsum(take.sum(0), 0)
    out = {"row_ptr": row_ptr, "col_idx": filled(e, -1, torch.int32), "val": filled(p[t, e], 0.0, torch.float64), "expert_ptr": expert_ptr,
           "token": filled(by_expert[:, 1], -1, torch.int32), "slot": filled(number[t, e], -1, torch.int32)}
    if case["backward"]:
        g = torch.zeros(T, E, dtype=torch.float64, device=DEVICE)
        g[t, e] = d["dval"][:n].double()
        out["dlogits"] = p * (g - (p * g).sum(1, keepdim=True))
    return out


def exact(case, seed):
    d, op = _inputs(case, seed), case["op"]
    if op == "route":
        return _exact_route(case, d)
    if op == "combine":
        n = int(d["row_ptr"][-1])
        row = torch.repeat_interleave(torch.arange(case["tokens"], device=DEVICE), d["row_ptr"][1:] - d["row_ptr"][:-1])
        slot = d["slot"][:n].long()
        val = d["val"][:n].double() if d["val"] is not None else torch.ones(n, dtype=torch.float64, device=DEVICE)
        y = d["y"].double()
        if not case["backward"]:
            return torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device=DEVICE).index_add_(0, row, val[:, None] * y[slot])
        dout = d["dout"].double()[row]
        dval = torch.zeros(case["tokens"] * case["k"], dtype=torch.float64, device=DEVICE)
        dval[:n] = (dout * y[slot]).sum(1)
        return {"dy": torch.zeros_like(y).index_copy_(0, slot, dout * val[:, None]), "dval": dval}
    if op == "grouped":
        ptr, x, dy = d["expert_ptr"].tolist(), d["x"].double(), d["dy"].double() if case["backward"] else None
        kn = case["layout"] == "kn"
        slots = d["token"].numel()
        first = torch.zeros(slots, case["inner"] if case["backward"] else case["outer"], dtype=torch.float64, device=DEVICE)
        dw = torch.zeros(d["w"].shape, dtype=torch.float64, device=DEVICE) if case["backward"] else None
        for e in range(case["experts"]):
            lo, hi = ptr[e], ptr[e + 1]
            if lo == hi:
                continue
            we = d["w"][e].double()
            we = we if kn else we.T            # [inner, outer]
            xe = x[d["token"][lo:hi].long()]
            if not case["backward"]:
                first[lo:hi] = torch.mm(xe, we)
            else:
                first[lo:hi] = torch.mm(dy[lo:hi], we.T)
                de = torch.mm(xe.T, dy[lo:hi])
                dw[e] = de if kn else de.T
        return {"dx": first, "dw": dw} if case["backward"] else first
    x = d["x"].double()
    y = torch.mm(x, d["w"].double().T)
    for a in range(case["adapters"]):
        at = torch.nonzero(d["ids"] == a)[:, 0]
        if at.numel():
            r = int(d["ranks"][a]) if d["ranks"] is not None else case["rank"]
            h = torch.mm(x[at], d["a"][a, :r].double().T)
            y[at] += d["scale"][a].double() * torch.mm(h, d["b"][a, :, :r].double().T)
    return y


def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == "route":
        T, E, k = case["tokens"], case["experts"], case["k"]
        nbytes = T * E * size + 16 * T * k + 8 * (T + E + 2)
        if case["backward"]:   # (gradient in, gradient out)
            nbytes += 4 * T * k + T * E * size
        return {"bytes": nbytes, "flops": 0}
    if op == "combine":
        live, k, D = case["tokens"] - case["pad"], case["k"], case["width"]
        lists = 8 * (case["tokens"] + 1) + live * k * (8 if case["weighted"] else 4)
        if case["backward"]:   # dout and y in, dy and dval out
            return {"bytes": lists + (case["tokens"] * (1 + k) * D + live * k * D) * size + 4 * case["tokens"] * k, "flops": 3 * live * k * D}
        return {"bytes": lists + (live * k + case["tokens"]) * D * size, "flops": 2 * live * k * D}
    K, N = case["inner"], case["outer"]
    if op == "grouped":
        live, k = case["tokens"] - case["pad"], case["k"]
        active = min(case["experts"] - case["closed"], live * k)
        lists = 8 * (case["experts"] + 1) + 4 * live * k
        if case["backward"]:   # dy, x and w in, dx and dw out
            nbytes = lists + size * (live * k * N + live * K + active * N * K + case["tokens"] * k * K + case["experts"] * N * K)
            return {"bytes": nbytes, "flops": 4 * live * k * K * N}
        return {"bytes": lists + size * (live * K + active * N * K + case["tokens"] * k * N), "flops": 2 * live * k * K * N}
    M, R = case["rows"], case["rank"]
    rank = R / 2 if case["ragged"] else R
    with_adapter = M * (1 - case["plain_rows"])
    requests = case["requests"] * (1 - case["plain_rows"])
    used = case["adapters"] * (1 - (1 - 1 / case["adapters"]) ** requests)
    return {"bytes": int(size * (M * K + N * K + M * N + used * rank * (K + N)) + 4 * M),
            "flops": int(2 * M * N * K + 2 * with_adapter * rank * (K + N))}
