"""The routed products from their definitions, in 64 bits on the CPU (NumPy).  Test infrastructure: nothing here is shared
with the GPU path."""
from __future__ import annotations

import numpy as np


def route(logits: np.ndarray, k: int, normalize: bool, lowest: float):
    """logits: float64 values of the type whose lowest finite value is `lowest`.  Returns a dict with the arrays of a routing
    matrix (padded to tokens * k as the library does), the dense weights p [tokens, experts] and the probabilities
    the weights come from."""
    T, E = logits.shape
    p = np.zeros((T, E))
    prob = np.zeros((T, E))
    rows = []
    for t in range(T):
        x = logits[t]
        open_ = [e for e in range(E) if not np.isnan(x[e]) and x[e] > lowest]
        value = {e: min(x[e], -lowest) for e in open_}
        taken = sorted(open_, key=lambda e: (-value[e], e))[:k]
        over = taken if normalize else open_
        if over:
            top = max(value.values())
            w = {e: np.exp(value[e] - top) for e in open_}
            total = sum(w[e] for e in over)
            for e in over:
                prob[t, e] = w[e] / total
            for e in taken:
                p[t, e] = prob[t, e]
        rows.append(sorted(taken))
    n = sum(len(r) for r in rows)
    out = {"row_ptr": np.cumsum([0] + [len(r) for r in rows]), "col_idx": np.full(T * k, -1), "val": np.zeros(T * k),
           "token": np.full(T * k, -1), "slot": np.full(T * k, -1)}
    entries = [(e, t) for t, r in enumerate(rows) for e in r]
    by_expert = sorted(range(n), key=lambda i: entries[i])
    out["expert_ptr"] = np.cumsum([0] + [sum(1 for e, _ in entries if e == c) for c in range(E)])
    for i, (e, t) in enumerate(entries):
        out["col_idx"][i], out["val"][i] = e, p[t, e]
    for s, i in enumerate(by_expert):
        out["slot"][i], out["token"][s] = s, entries[i][1]
    out["p"], out["prob"] = p, prob
    return out


def route_backward(r: dict, dval: np.ndarray, normalize: bool):
    T, E = r["p"].shape
    out = np.zeros((T, E))
    for t in range(T):
        lo, hi = r["row_ptr"][t], r["row_ptr"][t + 1]
        g = np.zeros(E)
        for i in range(lo, hi):
            g[r["col_idx"][i]] = dval[i]
        # softmax over the support of prob: J^T g with g zero at columns not taken
        out[t] = r["prob"][t] * (g - (r["prob"][t] * g).sum())
    return out


def combine(row_ptr, slot, val, y):
    """(out, sum of magnitudes)."""
    T = len(row_ptr) - 1
    out, mag = np.zeros((T, y.shape[1])), np.zeros((T, y.shape[1]))
    for t in range(T):
        for p in range(row_ptr[t], row_ptr[t + 1]):
            out[t] += val[p] * y[slot[p]]
            mag[t] += abs(val[p]) * np.abs(y[slot[p]])
    return out, mag


def combine_backward(row_ptr, slot, val, dout, y):
    """(dy, dval, magnitudes of dval)."""
    dy, dval, mag = np.zeros_like(y), np.zeros(len(slot)), np.zeros(len(slot))
    for t in range(len(row_ptr) - 1):
        for p in range(row_ptr[t], row_ptr[t + 1]):
            dy[slot[p]] = val[p] * dout[t]
            dval[p] = (dout[t] * y[slot[p]]).sum()
            mag[p] = np.abs(dout[t] * y[slot[p]]).sum()
    return dy, dval, mag


def grouped(group_ptr, x, w, rows=None):
    """y[s] = x[rows[s]] w_e^T, w [experts, outer, inner]; (y, magnitudes).  x has one row a slot where rows is None."""
    n = len(rows) if rows is not None else x.shape[0]
    y, mag = np.zeros((n, w.shape[1])), np.zeros((n, w.shape[1]))
    for e in range(len(group_ptr) - 1):
        for s in range(group_ptr[e], group_ptr[e + 1]):
            r = s if rows is None else rows[s]
            if 0 <= r < x.shape[0]:
                y[s] = w[e] @ x[r]
                mag[s] = np.abs(w[e]) @ np.abs(x[r])
    return y, mag


def grouped_weight_grad(group_ptr, dy, x, rows=None):
    """dw_e = sum dy[s]^T x[rows[s]]; (dw, magnitudes)."""
    E = len(group_ptr) - 1
    dw = np.zeros((E, dy.shape[1], x.shape[1]))
    mag = np.zeros_like(dw)
    for e in range(E):
        for s in range(group_ptr[e], group_ptr[e + 1]):
            r = s if rows is None else rows[s]
            if 0 <= r < x.shape[0]:
                dw[e] += np.outer(dy[s], x[r])
                mag[e] += np.outer(np.abs(dy[s]), np.abs(x[r]))
    return dw, mag


def adapter(x, w, a, b, ids, ranks=None, scale=None):
    """y[m] = x[m] w^T + scale (x[m] a_i^T) b_i^T; (y, magnitudes)."""
    y, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    for m, i in enumerate(ids):
        if 0 <= i < a.shape[0]:
            r = a.shape[1] if ranks is None else int(ranks[i])
            c = 1.0 if scale is None else float(scale[i])
            h, hm = a[i, :r] @ x[m], np.abs(a[i, :r]) @ np.abs(x[m])
            y[m] += c * (b[i, :, :r] @ h)
            mag[m] += abs(c) * (np.abs(b[i, :, :r]) @ hm)
    return y, mag
