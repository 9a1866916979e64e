"""The activation side in 64 bits (numpy): the 8-bit form, norm joins and their gradients, weight gradients.

Codes are found by going through all of them, scales by trying them upwards, so that nothing here shares a bit trick or an order of
operations with the kernels.  Pinned by hand-worked blocks, by neighbours on the number line and by differences in
tests/test_oracle_activations.py.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
I8, F8 = 0, 1
NONE, RMS, LAYER = 0, 1, 2
NO_GATE, CHANNEL, TOKEN, FULL = 0, 1, 2, 3


def code_values(fmt: int) -> np.ndarray:
    """What each of the 256 bytes stands for under scale 1; NaN for bytes that no encoder writes."""
    out = np.full(256, np.nan)
    for c in range(256):
        if fmt == I8:
            v = c - 256 if c >= 128 else c
            if v != -128:
                out[c] = v / 64
        else:
            sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
            if not (e == 15 and m == 7):
                out[c] = sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


def _round(x: np.ndarray, fmt: int) -> np.ndarray:
    """To the nearest of the format's numbers continued without an upper end, ties to the one whose last digit is even."""
    a = np.abs(x)
    if fmt == I8:
        step = np.full_like(a, 1 / 64)
    else:
        e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0))), -6)
        e = np.where(2.0 ** e > a, e - 1, e)
        e = np.where(2.0 ** (e + 1) <= a, e + 1, e)
        step = 2.0 ** (np.maximum(e, -6) - 3)
    return np.copysign(np.rint(a / step) * step, x)


LARGEST = {I8: 127 / 64, F8: 448.0}


def encode(x: np.ndarray, fmt: int):
    """x [rows, cols] -> (codes, scales), both uint8."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    values = code_values(fmt)
    q, scale = np.zeros((rows, cols), np.uint8), np.zeros((rows, nb), np.uint8)
    order = np.argsort(values[~np.isnan(values)], kind="stable")
    codes = np.arange(256, dtype=np.uint8)[~np.isnan(values)][order]
    sorted_values = values[codes]
    for r in range(rows):
        for b in range(nb):
            v = x[r, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
            if not np.all(np.isfinite(v)):
                scale[r, b] = 255
                continue
            top = np.max(np.abs(v))
            s = max(0, int(np.floor(np.log2(top))) + 127 - 12) if top > 0 else 0   # too small by far; then upwards
            while s < 254 and _round(np.array([top / 2.0 ** (s - 127)]), fmt)[0] > LARGEST[fmt]:
                s += 1
            scale[r, b] = s
            w = np.clip(_round(v / 2.0 ** (s - 127), fmt), -LARGEST[fmt], LARGEST[fmt])
            at = codes[np.searchsorted(sorted_values, w)]
            at = np.where(w == 0, np.where(np.signbit(w) & (fmt == F8), 128, 0), at)
            q[r, b * BLOCK:(b + 1) * BLOCK] = at
    return q, scale


def decode(q: np.ndarray, scale: np.ndarray, fmt: int) -> np.ndarray:
    m = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return code_values(fmt)[q] * np.repeat(m, BLOCK, axis=1)[:, :q.shape[1]]


def hat(v: np.ndarray, kind: int, eps: float):
    if kind == NONE:
        return v, np.ones(v.shape[0])
    c = v - v.mean(axis=1, keepdims=True) if kind == LAYER else v
    r = 1 / np.sqrt((c * c).mean(axis=1) + eps)
    return c * r[:, None], r


def join_forward(x, branch, scale, gate, pre, post):
    """pre, post: (kind, eps, weight or 1, bias or 0).  gate broadcasts.  Returns y, n, hat1, r1, hat2, r2 (None without a branch)."""
    y, h2, r2 = scale * x, None, None
    if branch is not None:
        h2, r2 = hat(branch, post[0], post[1])
        y = y + gate * (h2 * post[2] + post[3])
    h1, r1 = hat(y, pre[0], pre[1])
    return y, h1 * pre[2] + pre[3], h1, r1, h2, r2


def through(t, h, r, kind):
    if kind == NONE:
        return t
    u = t - h * (t * h).mean(axis=1, keepdims=True)
    if kind == LAYER:
        u = u - t.mean(axis=1, keepdims=True)
    return r[:, None] * u


def join_backward(dn, dy, scale, gate, gate_kind, pre, post, h1, r1, h2, r2):
    """Gradients by name; h1, h2: the normalised tensors as they were kept."""
    out = {}
    D = dy + through(dn * pre[2], h1, r1, pre[0])
    out["dx"] = scale * D
    out["dpre_weight"], out["dpre_bias"] = (dn * h1).sum(0), dn.sum(0)
    out["D"] = D
    if h2 is not None:
        g = D * (h2 * post[2] + post[3])
        out["dgate"] = {NO_GATE: None, CHANNEL: g.sum(0, keepdims=True), TOKEN: g.sum(1, keepdims=True), FULL: g}[gate_kind]
        dc = gate * D
        out["dbranch"] = through(dc * post[2], h2, r2, post[0])
        out["dpost_weight"], out["dpost_bias"] = (dc * h2).sum(0), dc.sum(0)
    return out


def weight_grad(dy, kept, weight, bias, offsets=None):
    """dw, db; with offsets one of each per group, offsets clipped into the tokens and counting up."""
    z = kept * weight + bias
    if offsets is None:
        return dy.T @ z, dy.sum(0)
    t, dw, db = len(dy), [], []
    for a, b in zip(offsets[:-1], offsets[1:]):
        a = min(max(int(a), 0), t)
        b = min(max(int(b), a), t)
        dw.append(dy[a:b].T @ z[a:b])
        db.append(dy[a:b].sum(0))
    return np.stack(dw), np.stack(db)
