"""Oracle: block tables, slot map and free list of a growing batch, request after
request with plain lists (test infrastructure; InferLog section 2.1.2: KV blocks
are allocated as tokens come and freed when a request ends)."""
from __future__ import annotations

BLOCK = 16
NO_BLOCKS, TOO_LONG, TOO_MANY_ROWS, BAD_VALUE = 1, 2, 4, 8


def _blocks(n):
    return -(-n // BLOCK)


def extend_ref(tables, start, new, free, taken, num_blocks, max_rows):
    """Returns (tables, seq_lens, cu_q, cu_blocks, slots, taken, status)."""
    B, tables, mb = len(start), [list(t) for t in tables], len(tables[0]) if len(tables) else 1
    need = [_blocks(s + n) - _blocks(s) for s, n in zip(start, new)]
    status = 0
    if not 0 <= taken <= len(free) or any(s < 0 or n < 0 for s, n in zip(start, new)):
        status |= BAD_VALUE
    if any(s + n > BLOCK * mb for s, n in zip(start, new)):
        status |= TOO_LONG
    if taken + sum(need) > len(free):
        status |= NO_BLOCKS
    if sum(new) > max_rows:
        status |= TOO_MANY_ROWS
    if status:
        return tables, list(start), [0] * (B + 1), [0] * (B + 1), [-1] * max_rows, taken, status
    seq, cu_q, cu_b, slots, at = [], [0], [0], [], taken
    for r in range(B):
        for j in range(_blocks(start[r]), _blocks(start[r] + new[r])):
            tables[r][j] = free[at]
            at += 1
        for p in range(start[r], start[r] + new[r]):
            b = tables[r][p // BLOCK]
            slots.append(b * BLOCK + p % BLOCK if 0 <= b < num_blocks else -1)
        seq.append(start[r] + new[r])
        cu_q.append(len(slots))
        cu_b.append(at - taken)
    return tables, seq, cu_q, cu_b, slots + [-1] * (max_rows - len(slots)), at, 0


def release_ref(tables, first, seq, free, taken):
    """Returns (free, cu_blocks, taken, status)."""
    B, free, mb = len(first), list(free), len(tables[0]) if len(tables) else 1
    gone, cu, status = [], [0], 0
    for r in range(B):
        gone += [tables[r][j] if 0 <= j < mb else None for j in range(first[r], _blocks(seq[r]))] if first[r] >= 0 else []
        cu.append(len(gone))
    if not 0 <= taken <= len(free) or any(f < 0 or s < 0 for f, s in zip(first, seq)):
        status |= BAD_VALUE
    if any(s > BLOCK * mb for s in seq):
        status |= TOO_LONG
    if status & BAD_VALUE:  # (counts of negative values mean nothing)
        return free, [0] * (B + 1), taken, status
    if len(gone) > taken:
        status |= NO_BLOCKS
    if status:
        return free, [0] * (B + 1), taken, status
    free[taken - len(gone):taken] = gone
    return free, cu, taken - len(gone), 0
