"""CPU oracle of the operators around a paged cache, float64.

TEST INFRASTRUCTURE ONLY (see expert_oracle.py): nothing in the product path may import this file.

What it computes, from the definitions (the paper names the prefix caches, not their paging; the norm is the expert's, with gain 1 +
gamma, the rotation is the expert's, of channels j and j + dh / 2):

* ``heads``: x [T, H, dh] -> norm (gain None: none) and rotation by a (cos, sin) table at the tokens' positions;
* ``slots``: rows of the planes that hold a request's cached tokens;
* ``append``: the pool after the new tokens' keys and values have been written;
* ``attend``: attention of the new tokens over their requests' cached tokens, keys [0, limit) of each;
* ``pack``: the cached tokens as a ragged cache.

Beside a result, ``heads`` and ``attend`` return the sizes by which the rounding of a fp32 computation is bounded."""
from __future__ import annotations

import numpy as np


def heads(x, gain, eps, table, positions):
    """Returns (y, the size of the terms of each y: |a cos| + |b sin|)."""
    x = np.asarray(x, dtype=np.float64)
    half = x.shape[-1] // 2
    if gain is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * (1.0 + np.asarray(gain, dtype=np.float64))
    if table is None:
        return x, np.abs(x)
    t = np.asarray(table, dtype=np.float64)[np.asarray(positions)]
    c, s = t[:, None, :, 0], t[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    y = np.concatenate([a * c - b * s, b * c + a * s], axis=-1)
    size = np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], axis=-1)
    return y, size


def slots(table_row, page_size, n):
    return np.array([int(table_row[t // page_size]) * page_size + t % page_size for t in range(n)], dtype=np.int64)


def append(plane_k, plane_v, k, v, cu, kv_lens, table, page_size):
    """Planes [rows, Hkv, dh] of one layer; writes the new tokens' rows (already normed and rotated)."""
    plane_k, plane_v = plane_k.copy(), plane_v.copy()
    for b, kv in enumerate(kv_lens):
        n = int(cu[b + 1] - cu[b])
        rows = slots(table[b], page_size, int(kv))[int(kv) - n:]
        plane_k[rows], plane_v[rows] = k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]]
    return plane_k, plane_v


def limits(n, kv, causal, prefix):
    if not causal:
        return np.full(n, kv, dtype=np.int64)
    return np.clip(np.maximum(kv - n + 1 + np.arange(n), prefix), 0, kv)


def attend(q, plane_k, plane_v, cu, kv_lens, table, page_size, causal, prefix_lens=None, scale=None):
    """q [T, Hq, dh], planes [rows, Hkv, dh].  Returns (out, weights times |v|, largest sum of |q k| scale of a row); rows of no request
    are NaN."""
    T, Hq, dh = q.shape
    Hkv = plane_k.shape[1]
    scale = 1.0 / np.sqrt(dh) if scale is None else scale
    out, size, big = np.full((T, Hq, dh), np.nan), np.full((T, Hq, dh), np.nan), np.full((T, Hq, 1), np.nan)
    for b, kv in enumerate(kv_lens):
        n, kv = int(cu[b + 1] - cu[b]), int(kv)
        rows = slots(table[b], page_size, kv)
        lim = limits(n, kv, causal, 0 if prefix_lens is None else int(prefix_lens[b]))
        for h in range(Hq):
            g = h // (Hq // Hkv)
            k, v = plane_k[rows, g].astype(np.float64), plane_v[rows, g].astype(np.float64)
            for i in range(n):
                t, m = int(cu[b]) + i, int(lim[i])
                if m == 0:
                    out[t, h], size[t, h], big[t, h] = 0.0, 0.0, 0.0
                    continue
                x = q[t, h].astype(np.float64)
                s = k[:m] @ x * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h], size[t, h] = w @ v[:m], w @ np.abs(v[:m])
                big[t, h] = (np.abs(k[:m]) @ np.abs(x)).max() * scale
    return out, size, big


def pack(planes, kv_lens, table, page_size):
    """planes [L, 2, rows, Hkv, dh] -> ([L, 2, sum, Hkv, dh], cu)."""
    rows = [slots(table[b], page_size, int(n)) for b, n in enumerate(kv_lens)]
    cu = np.concatenate([[0], np.cumsum(kv_lens)]).astype(np.int32)
    return planes[:, :, np.concatenate(rows)] if cu[-1] else planes[:, :, :0], cu
