"""The token side in 64 bits (numpy): sorting by id, lookup and its gradients, products per group, the dropout mask.

Everything goes position by position or group by group, in loops and whole-number arithmetic of Python, so that nothing here shares an
order of operations with the kernels.  Pinned by hand-worked cases, by differences and by the generator's published outputs in
tests/test_oracle_tokens.py.
"""
from __future__ import annotations

import numpy as np


def sort_tokens(ids, rows: int, per_token: int = 1):
    """(order, offsets, place, token) of a flat list of ids."""
    ids = [int(i) for i in ids]
    found = [[] for _ in range(rows + 1)]
    for p, i in enumerate(ids):
        found[i if 0 <= i < rows else rows].append(p)
    order = [p for row in found for p in row]
    offsets = np.concatenate([[0], np.cumsum([len(row) for row in found[:rows]])])
    place = np.full(len(ids), -1)
    for i, p in enumerate(order[:offsets[-1]]):
        place[p] = i
    order = np.asarray(order, dtype=np.int64)
    return order, offsets.astype(np.int64), place.astype(np.int64), order // per_token


def lookup(ids, table, scale=1.0, weights=None):
    """(y, sum of the terms' sizes) for ids [tokens, per_token]."""
    tokens, per = ids.shape
    y, size = np.zeros((tokens, table.shape[1])), np.zeros((tokens, table.shape[1]))
    for t in range(tokens):
        for j in range(per):
            if 0 <= ids[t, j] < len(table):
                part = (1.0 if weights is None else weights[t, j]) * table[ids[t, j]] * scale
                y[t] += part
                size[t] += np.abs(part)
    return y, size


def lookup_gradients(ids, dy, rows: int, table=None, scale=1.0, weights=None):
    """(dtable, its terms' sizes, dweights, its terms' sizes); the last two None without a table."""
    tokens, per = ids.shape
    dtable, size = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1]))
    dw = None if table is None else np.zeros((tokens, per))
    dw_size = None if table is None else np.zeros((tokens, per))
    for t in range(tokens):
        for j in range(per):
            r = int(ids[t, j])
            if 0 <= r < rows:
                part = scale * (1.0 if weights is None else weights[t, j]) * dy[t]
                dtable[r] += part
                size[r] += np.abs(part)
                if table is not None:
                    dw[t, j], dw_size[t, j] = scale * np.sum(dy[t] * table[r]), abs(scale) * np.sum(np.abs(dy[t] * table[r]))
    return dtable, size, dw, dw_size


def grouped_product(x, w, offsets, bias=None, transposed=False, y=None):
    """(y, the terms' sizes); w [groups, out, in] or, transposed, [groups, in, out].  Rows in no group are those of the given y."""
    out = w.shape[2] if transposed else w.shape[1]
    y = np.zeros((len(x), out)) if y is None else y.copy()
    size = np.zeros((len(x), out))
    for g in range(len(w)):
        m = w[g] if transposed else w[g].T
        a, b = min(max(int(offsets[g]), 0), len(x)), min(max(int(offsets[g + 1]), 0), len(x))
        if a < b:
            y[a:b] = x[a:b] @ m + (0.0 if bias is None else bias[g])
            size[a:b] = np.abs(x[a:b]) @ np.abs(m) + (0.0 if bias is None else np.abs(bias[g]))
    return y, size


def philox(counter, key):
    """The four words of Philox4x32 of ten rounds, as whole numbers (Salmon et al., SC 2011)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b % 2 ** 32, (a >> 32) ^ c[3] ^ k[1], a % 2 ** 32]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def dropout_bits(rows: int, cols: int, seed: int, layer: int = 0, first_row: int = 0):
    """The 16 random bits of each element."""
    u = np.zeros((rows, cols), dtype=np.int64)
    for r in range(rows):
        row = first_row + r
        for block in range(-(-cols // 8)):
            words = philox((block, row % 2 ** 32, row >> 32, layer), (seed % 2 ** 32, (seed >> 32) % 2 ** 32))
            for i in range(min(8, cols - 8 * block)):
                u[r, 8 * block + i] = (words[i // 2] >> (16 * (i % 2))) % 65536
    return u


def dropout(x, p: float, seed: int, layer: int = 0, first_row: int = 0, residual=None):
    bound = int(np.floor(p * 65536 + 0.5))
    kept = dropout_bits(*x.shape, seed, layer, first_row) >= bound
    y = np.where(kept, x * (65536 / (65536 - bound) if bound < 65536 else 0.0), 0.0)
    return y if residual is None else y + residual
