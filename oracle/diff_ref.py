"""Oracle: dense float64 differential attention of one request (test infrastructure).

Each head is the difference of two causal softmax maps over one set of values
(the suffix queries of a prompt over its reused and new KV, InferLog section
2.1.2): with the two maps' parts of the D dimensions of q and k,

    A_m = softmax(scale q_m k_m^T),  y = (A_1 - lam_h A_2) V,
    out = out_scale * w * y / sqrt(mean(y^2) + eps)     (w None: out_scale * y).

The parts are the halves of D (layout "halves"), or, so that rotate-half pairs
(i, i + D/2) stay within a map, the quarters 0 and 2 against 1 and 3 ("rope").
It never sees a paged pool or a block table.
"""
from __future__ import annotations

import numpy as np


def map_dims(D: int, layout: str, m: int) -> np.ndarray:
    q = np.arange(D).reshape(4, D // 4)
    return np.concatenate([q[2 * m], q[2 * m + 1]] if layout == "halves" else [q[m], q[2 + m]])


def diff_attention_ref(q, k, v, scale, lam, w=None, eps=1e-5, out_scale=1.0, layout="halves", with_size=False):
    """q: [S, Hq, D]; k, v: [L, Hkv, D], S <= L; lam: [Hq]; w: [D] or None.  Returns
    float64 [S, Hq, D]; with_size: also sum_j (A_1 + |lam| A_2)_j |v_j| under the same
    factors, the size of the terms that the output is a difference of."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    lam = np.asarray(lam, dtype=np.float64)
    S, Hq, D = q.shape
    L, Hkv, _ = k.shape
    G = Hq // Hkv
    seen = np.arange(L)[None, :] <= (L - S + np.arange(S))[:, None]
    out, size = np.empty((S, Hq, D)), np.empty((S, Hq, D))
    for h in range(Hq):
        maps = []
        for m in (0, 1):
            d = map_dims(D, layout, m)
            z = np.where(seen, scale * (q[:, h][:, d] @ k[:, h // G][:, d].T), -np.inf)
            e = np.exp(z - z.max(axis=1, keepdims=True))
            maps.append(e / e.sum(axis=1, keepdims=True))
        y = (maps[0] - lam[h] * maps[1]) @ v[:, h // G]
        f = np.full((S, D), float(out_scale))
        if w is not None:
            f = f * np.asarray(w, dtype=np.float64) / np.sqrt((y * y).mean(axis=1, keepdims=True) + eps)
        out[:, h] = y * f
        if with_size:
            size[:, h] = ((maps[0] + abs(lam[h]) * maps[1]) @ np.abs(v[:, h // G])) * np.abs(f)
    return (out, size) if with_size else out
