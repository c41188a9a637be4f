"""Pins of the tree and fork oracle: hand-worked trees, closed forms, the causal chain
against the pinned attention oracle, and holders counted block by block."""
import numpy as np
import pytest

from oracle import tree_ref
from oracle.attn_ref import prefill_attention_ref

# node:     0   1  2  3  4  5  6
PARENTS = [-1, 0, 0, 1, 1, 2, 4]
TOKENS = [50, 7, 8, 9, 7, 9, 3]


def test_ancestors_of_a_hand_worked_tree():
    assert tree_ref.ancestors(PARENTS) == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 4], [0, 2, 5], [0, 1, 4, 6]]
    masks, pos = tree_ref.masks_ref(PARENTS, 100, 1)
    assert [m[0] for m in masks] == [1, 3, 5, 11, 19, 37, 83] and pos == [100, 101, 101, 102, 102, 102, 103]


def test_masks_of_chains_stars_padding_and_further_words():
    n = 70
    masks, pos = tree_ref.masks_ref([i - 1 for i in range(n)], 0, 2)
    assert [m[0] | m[1] << 64 for m in masks] == [(1 << (i + 1)) - 1 for i in range(n)] and pos == list(range(n))
    masks, pos = tree_ref.masks_ref([-1] + [0] * 9, 5, 1)
    assert [m[0] for m in masks] == [1] + [1 | 1 << i for i in range(1, 10)] and pos == [5] + [6] * 9
    masks, pos = tree_ref.masks_ref([-1, 1, 5, -2, 0], 3, 1)  # parents that are not before their node
    assert [m[0] for m in masks] == [1, 2, 4, 8, 17] and pos == [3, 3, 3, 3, 4]
    masks, _ = tree_ref.masks_ref([i - 1 for i in range(66)], 0, 1)
    assert masks[63] == [(1 << 64) - 1] and masks[64] == masks[65] == [0]


def test_accepted_paths_of_a_hand_worked_tree():
    t = [7, 7, 1, 1, 3, 1, 77]
    assert tree_ref.accept_ref(PARENTS, TOKENS, t) == ([0, 1, 4, 6], 77)
    assert tree_ref.accept_ref(PARENTS, TOKENS, [8] + t[1:]) == ([0, 2], 1)
    assert tree_ref.accept_ref(PARENTS, TOKENS, [99] + t[1:]) == ([0], 99)
    assert tree_ref.accept_ref(PARENTS, TOKENS, t, root_target=50) == ([0, 1, 4, 6], 77)
    assert tree_ref.accept_ref(PARENTS, TOKENS, t, root_target=51) == ([], 51)
    assert tree_ref.accept_ref([-1, 0, 0], [1, 2, 2], [2, 5, 6]) == ([0, 1], 5)  # twins: the first
    assert tree_ref.accept_ref([], [], []) == ([], -1) and tree_ref.accept_ref([-2], [1], [1]) == ([], -1)


def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(12, 2, 8)), rng.normal(size=(12, 2, 8))
    out, mag = tree_ref.tree_attention_ref(q, k, v, 0.3, np.tril(np.ones((5, 5))))
    assert np.abs(out - prefill_attention_ref(q, k, v, 0.3)).max() < 1e-12
    assert (mag >= np.abs(out) - 1e-12).all()


def test_a_branch_is_the_sequence_of_its_path():
    # a node's row is the last row of the plain sequence context + its ancestors
    rng = np.random.default_rng(1)
    n = len(PARENTS)
    q, k, v = rng.normal(size=(n, 2, 8)), rng.normal(size=(6 + n, 1, 8)), rng.normal(size=(6 + n, 1, 8))
    lines = tree_ref.ancestors(PARENTS)
    seen = np.array([[j in line for j in range(n)] for line in lines])
    out, _ = tree_ref.tree_attention_ref(q, k, v, 0.5, seen)
    for i, line in enumerate(lines):
        keys = list(range(6)) + [6 + j for j in line]
        assert np.abs(out[i] - prefill_attention_ref(q[i:i + 1], k[keys], v[keys], 0.5)[0]).max() < 1e-12


def test_a_row_without_keys_is_zero_and_one_key_gives_its_value():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(3, 2, 4)), rng.normal(size=(3, 2, 4)), rng.normal(size=(3, 2, 4))
    out, _ = tree_ref.tree_attention_ref(q, k, v, 1.0, [[0, 0, 0], [0, 1, 0], [1, 0, 1]])
    assert (out[0] == 0).all() and np.allclose(out[1], v[1])


def test_forks_by_hand():
    # row 0: 40 tokens in blocks 9 (the cache's), 20, 21; rows 1 and 2 become forks; row 3 stays
    tables = [[9, 20, 21, -1], [5, 5, 5, 5], [-1] * 4, [22, -1, -1, -1]]
    t, n, h, src, dst, taken, st = tree_ref.fork_ref(tables, [40, 0, 0, 16], [0, 0, 0, 3], [0] * 10, 20,
                                                     list(range(20, 30)), 3, 30)
    assert t == [[9, 20, 21, -1], [9, 20, 23, -1], [9, 20, 24, -1], [22, -1, -1, -1]] and n == [40, 40, 40, 16]
    assert h == [2] + [0] * 9 and (src, dst) == ([-1, 21, 21, -1], [-1, 23, 24, -1]) and (taken, st) == (5, 0)
    # the source ends first, its full block goes on
    free = list(range(20, 30))
    h, free, taken, st = tree_ref.release_shared_ref(t, [40, 0, 0, 0], h, 20, free, taken, 30)
    assert h == [1] + [0] * 9 and free[4] == 21 and (taken, st) == (4, 0)
    h, free, taken, st = tree_ref.release_shared_ref(t, [0, 40, 40, 0], h, 20, free, taken, 30)
    assert h == [0] * 10 and free[1:5] == [20, 23, 24, 21] and (taken, st) == (1, 0)


@pytest.mark.parametrize("seed", range(5))
def test_holds_are_the_holders_beyond_the_first(seed):
    rng = np.random.default_rng(seed)
    B, mb, first, nb = 12, 8, 10, 200
    free, taken, holds = list(range(first, nb)), 0, [0] * (nb - first)
    tables, lens = [[-1] * mb for _ in range(B)], [0] * B
    live = {0, 1, 2}
    for r in live:
        lens[r] = int(rng.integers(1, 16 * mb + 1))
        for j in range(-(-lens[r] // 16)):
            tables[r][j] = free[taken] if j else r
            taken += j > 0
    for _ in range(30):
        if rng.random() < 0.5 and len(live) < B:
            src = list(range(B))
            for r in set(range(B)) - live:
                if rng.random() < 0.6:
                    src[r] = int(rng.choice(sorted(live)))
            tables, lens, holds, _, _, taken, st = tree_ref.fork_ref(tables, lens, src, holds, first, free, taken, nb)
            live |= {r for r in range(B) if src[r] != r}
        else:
            ended = {r for r in live if r != min(live) and rng.random() < 0.4}
            holds, free, taken, st = tree_ref.release_shared_ref(tables, [lens[r] if r in ended else 0 for r in range(B)],
                                                                 holds, first, free, taken, nb)
            live -= ended
        assert st == 0
        count = {}
        for r in live:
            for b in tables[r][:-(-lens[r] // 16)]:
                count[b] = count.get(b, 0) + 1
        assert all(holds[b - first] == max(count.get(b, 0) - 1, 0) for b in range(first, nb))
        assert sorted(free[taken:] + [b for b in count if b >= first]) == list(range(first, nb))
