"""Losses of a router and matrices in microscaled four bits from their definitions, in 64 bits on the CPU (NumPy).  Test infrastructure: nothing here is
shared with the GPU path."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def balance(logits: np.ndarray, counts: np.ndarray, lowest: float):
    """logits: float64 values of the type whose lowest finite value is `lowest`.  loss, prob, rows, and p [tokens, experts], lse [tokens] (0 for a row
    without an open logit)."""
    T, E = logits.shape
    p, lse = np.zeros((T, E)), np.zeros(T)
    rows = 0
    for t in range(T):
        open_ = ~np.isnan(logits[t]) & (logits[t] > lowest)
        if not open_.any():
            continue
        rows += 1
        x = np.minimum(logits[t][open_], -lowest)
        top = x.max()
        e = np.exp(x - top)
        p[t, open_] = e / e.sum()
        lse[t] = top + np.log(e.sum())
    n = counts.sum()
    prob = p.sum(0) / rows if rows else np.zeros(E)
    even = E * float((counts / n * prob).sum()) if n > 0 else 0.0
    with np.errstate(over="ignore"):
        size = float((lse ** 2).sum() / rows) if rows else 0.0
    return {"loss": np.array([even, size]), "prob": prob, "rows": rows, "p": p, "lse": lse}


def balance_backward(b: dict, counts: np.ndarray, rows: int, dloss):
    """(gradient of the logits, a bound of the magnitudes that it is the sum of)."""
    T, E = b["p"].shape
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    share = counts / counts.sum() if counts.sum() > 0 else np.zeros(E)
    for t in range(T):
        p = b["p"][t]
        if rows == 0:
            continue
        met = float((p * share).sum())
        even, size = dloss[0] * E / rows, 2 * dloss[1] / rows * b["lse"][t]
        out[t] = p * (even * (share - met) + size)
        mag[t] = p * (abs(even) * (share + met) + abs(size))
    return out, mag


def quantize(x: np.ndarray):
    """x: float64 [rows, inner].  Codes [rows, blocks * 32] (0 .. 15) and scales [rows, blocks]."""
    rows, inner = x.shape
    blocks = (inner + 31) // 32
    codes, scales = np.zeros((rows, blocks * 32), dtype=np.int64), np.zeros((rows, blocks), dtype=np.int64)
    middle = (E2M1[1:] + E2M1[:-1]) / 2
    for i in range(rows):
        for b in range(blocks):
            part = x[i, b * 32:(b + 1) * 32]
            if not np.isfinite(part).all():
                scales[i, b] = 255
                continue
            top = np.abs(part).max()
            e = 0 if top == 0 else max(int(np.frexp(top)[1]) - 3, -127)
            scales[i, b] = e + 127
            v = np.abs(part) / 2.0 ** e
            code = np.searchsorted(middle, v, side="left")      # (ties: to the code below ...)
            tie = np.isin(v, middle) & (code % 2 == 1)
            code = np.where(tie, code + 1, code)                # (... or the even one above)
            codes[i, b * 32:b * 32 + len(part)] = code + 8 * np.signbit(part)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray, inner: int):
    v = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes % 8]
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(unit, 32, axis=-1))[..., :inner]


def pack(codes: np.ndarray):
    return (codes[..., ::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(packed: np.ndarray):
    return np.stack([packed & 15, packed >> 4], axis=-1).reshape(*packed.shape[:-1], 2 * packed.shape[-1]).astype(np.int64)
