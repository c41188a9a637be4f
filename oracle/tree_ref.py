"""Oracle: trees of drafted tokens, node after node with plain lists, their attention in
float64 on dense K/V, and forked rows with explicit holders of every block (test
infrastructure; InferLog section 2.1.2: the newest tokens attend to the cached KV of
their context; blocks are shared by requests and freed when none holds them)."""
from __future__ import annotations

import numpy as np

BLOCK = 16
NO_BLOCKS, TOO_LONG, BAD_VALUE, NOT_HELD = 1, 2, 8, 16


def _blocks(n):
    return -(-n // BLOCK)


def ancestors(parents):
    """Per node the sorted list of itself and its ancestors (a parent outside [-1, i): itself alone)."""
    out = []
    for i, p in enumerate(parents):
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def masks_ref(parents, start, words):
    """(masks as lists of Python ints, 64 bits a word; positions) of one request."""
    masks, pos = [], []
    for i, line in enumerate(ancestors(parents)):
        if i >= 64 * words:
            masks.append([0] * words)
            pos.append(start)
            continue
        masks.append([sum(1 << (j - 64 * w) for j in line if j // 64 == w) for w in range(words)])
        pos.append(start + len(line) - 1)
    return masks, pos


def accept_ref(parents, tokens, targets, root_target=None):
    """(path, next token) of one request; root_target None: node 0 is the root."""
    n, path = len(parents), []
    if root_target is None:
        if n == 0 or parents[0] != -1:
            return [], -1
        path, want = [0], targets[0]
    else:
        want = root_target
    while True:
        last = path[-1] if path else -1
        child = [i for i in range(n) if parents[i] == last and -1 <= parents[i] < i and tokens[i] == want]
        if not child:
            return path, want
        path.append(child[0])
        want = targets[child[0]]


def tree_attention_ref(q, k, v, scale, seen):
    """q [S, Hq, D], k and v [L, Hkv, D], seen bool [S, S]: row i sees all keys before the last S and
    of those the ones of seen[i].  Returns (out, sum of weights times |v|), float64."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    S, Hq, D = q.shape
    L, Hkv, _ = k.shape
    vis = np.concatenate([np.ones((S, L - S), bool), np.asarray(seen, bool)], 1)
    kr, vr = np.repeat(k, Hq // Hkv, 1), np.repeat(v, Hq // Hkv, 1)
    s = np.where(vis[None], np.matmul(q.transpose(1, 0, 2), kr.transpose(1, 2, 0)) * scale, -np.inf)
    top = s.max(-1, keepdims=True, initial=-np.inf)
    with np.errstate(invalid="ignore"):
        p = np.where(vis[None], np.exp(s - top), 0.0)
    total = p.sum(-1, keepdims=True)
    p = p / np.where(total > 0, total, 1.0)
    out, mag = np.matmul(p, vr.transpose(1, 0, 2)), np.matmul(p, np.abs(vr).transpose(1, 0, 2))
    return out.transpose(1, 0, 2), mag.transpose(1, 0, 2)


def fork_ref(tables, lens, sources, holds, first_id, free, taken, num_blocks):
    """Returns (tables, lens, holds, copy_src, copy_dst, taken, status); holds: counts alone."""
    B, mb = len(lens), len(tables[0]) if len(tables) else 1
    status, ok = 0, [0 <= s < B for s in sources]
    if not 0 <= taken <= len(free) or not all(ok):
        status |= BAD_VALUE
    need = 0
    for r, s in enumerate(sources):
        if ok[r]:
            status |= BAD_VALUE if sources[s] != s or lens[s] < 0 else 0
            status |= TOO_LONG if lens[s] > BLOCK * mb else 0
            need += s != r and lens[s] % BLOCK != 0
    if taken + need > len(free):
        status |= NO_BLOCKS
    none = [-1] * B
    if status:
        return tables, lens, holds, none, none, taken, status
    tables, lens, holds, src, dst = [list(t) for t in tables], list(lens), list(holds), list(none), list(none)
    for r, s in enumerate(sources):
        if s == r:
            continue
        row = [-1] * mb
        for j in range(lens[s] // BLOCK):
            row[j] = tables[s][j]
            if first_id <= row[j] < num_blocks:
                holds[row[j] - first_id] += 1
        if lens[s] % BLOCK:
            j = lens[s] // BLOCK
            src[r], dst[r] = tables[s][j], free[taken]
            row[j] = free[taken]
            taken += 1
        tables[r], lens[r] = row, lens[s]
    return tables, lens, holds, src, dst, taken, 0


def release_shared_ref(tables, lens, holds, first_id, free, taken, num_blocks):
    """Returns (holds, free, taken, status); holds: counts alone."""
    mb = len(tables[0]) if len(tables) else 1
    status = 0
    if not 0 <= taken <= len(free) or any(n < 0 for n in lens):
        status |= BAD_VALUE
    if any(n > BLOCK * mb for n in lens):
        status |= TOO_LONG
    if status:
        return holds, free, taken, status
    left, gone = list(holds), []
    for r, n in enumerate(lens):
        for b in tables[r][:_blocks(n)]:
            if first_id <= b < num_blocks:
                left[b - first_id] -= 1
                if left[b - first_id] == -1:
                    gone.append(b)
                if left[b - first_id] < -1:
                    status |= NOT_HELD
    if len(gone) > taken:
        status |= NO_BLOCKS
    if status:
        return holds, free, taken, status
    for b in gone:
        left[b - first_id] = 0
    free = list(free)
    free[taken - len(gone):taken] = sorted(gone)
    return left, free, taken - len(gone), 0
