"""Pins of the differential-attention and growing-batch oracles (CPU)."""
import math

import numpy as np
import pytest

from oracle.attn_ref import prefill_attention_ref
from oracle.diff_ref import diff_attention_ref, map_dims
from oracle.rope_ref import rope
from oracle.tables_ref import BLOCK, extend_ref, release_ref


def rand(*shape, seed=0):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("layout", ["halves", "rope"])
def test_maps_split_the_dimensions(layout):
    for D in (64, 128):
        a, b = map_dims(D, layout, 0), map_dims(D, layout, 1)
        assert sorted([*a, *b]) == list(range(D)) and len(a) == len(b)
        if layout == "rope":  # rotation pairs stay within a map
            assert {(i + D // 2) % D for i in a} == set(a)


@pytest.mark.parametrize("layout", ["halves", "rope"])
def test_is_the_difference_of_two_ordinary_attentions(layout):
    S, L, Hq, Hkv, D = 3, 7, 4, 2, 8
    q, k, v, lam = rand(S, Hq, D), rand(L, Hkv, D, seed=1), rand(L, Hkv, D, seed=2), rand(Hq, seed=3)
    got = diff_attention_ref(q, k, v, 0.5, lam, layout=layout)
    both = []
    for m in (0, 1):  # the other map's dimensions zero
        keep = np.zeros(D)
        keep[map_dims(D, layout, m)] = 1
        both.append(prefill_attention_ref(q * keep, k, v, 0.5))
    np.testing.assert_allclose(got, both[0] - lam[None, :, None] * both[1], atol=1e-12)


def test_brute_force_with_norm():
    S, L, D = 2, 3, 4
    q, k, v, lam, w = rand(S, 1, D), rand(L, 1, D, seed=1), rand(L, 1, D, seed=2), [0.7], rand(D, seed=4)
    got = diff_attention_ref(q, k, v, 0.9, lam, w, eps=0.01, out_scale=0.3)
    for t in range(S):
        n, y = L - S + t + 1, [0.0] * D
        for m, sign in ((0, 1.0), (1, -0.7)):
            e = [math.exp(0.9 * sum(q[t, 0, 2 * m + i] * k[j, 0, 2 * m + i] for i in range(2))) for j in range(n)]
            for d in range(D):
                y[d] += sign * sum(e[j] * v[j, 0, d] for j in range(n)) / sum(e)
        rms = math.sqrt(sum(x * x for x in y) / D + 0.01)
        np.testing.assert_allclose(got[t, 0], [0.3 * w[d] * y[d] / rms for d in range(D)], atol=1e-12)


def test_equal_maps_cancel_and_one_key_gives_its_value():
    q, k, v = rand(2, 2, 8), rand(5, 1, 8, seed=1), rand(5, 1, 8, seed=2)
    q[..., 4:], k[..., 4:] = q[..., :4], k[..., :4]
    assert np.abs(diff_attention_ref(q, k, v, 1.0, [1.0, 1.0])).max() < 1e-12
    np.testing.assert_allclose(diff_attention_ref(q[:1], k[:1], v[:1], 1.0, [0.25, 2.0]),
                               v[:1] * np.array([0.75, -1.0])[None, :, None], atol=1e-12)


def test_rope_layout_is_a_rotation_of_each_map():
    # rotating whole heads with the angles of a map twice, then the pair layout, is
    # rotating each map's D/2 dimensions by themselves, then the halves
    D, L = 16, 6
    ang = 100.0 ** (-np.arange(D // 4) / (D // 4))
    q, k, v = rand(L, 1, D), rand(L, 1, D, seed=1), rand(L, 1, D, seed=2)
    pos = np.arange(L)
    whole = [rope(x, pos, np.concatenate([ang, ang])) for x in (q, k)]
    a = diff_attention_ref(*whole, v, 0.4, [0.6], layout="rope")
    order = np.concatenate([map_dims(D, "rope", 0), map_dims(D, "rope", 1)])
    own = [np.concatenate([rope(x[..., map_dims(D, "rope", m)], pos, ang) for m in (0, 1)], axis=-1)
           for x in (q, k)]
    np.testing.assert_allclose(own[0], whole[0][..., order], atol=1e-12)
    np.testing.assert_allclose(a, diff_attention_ref(*own, v, 0.4, [0.6]), atol=1e-12)


def test_tables_by_hand():
    t = [[7, 8, -1], [9, -1, -1], [-1, -1, -1]]
    tables, seq, cu, cb, slots, taken, status = extend_ref(t, [20, 16, 0], [13, 1, 0], [5, 4, 3, 2], 1, 10, 16)
    assert tables == [[7, 8, 4], [9, 3, -1], [-1, -1, -1]] and seq == [33, 17, 0] and status == 0
    assert cu == [0, 13, 14, 14] and cb == [0, 1, 2, 2] and taken == 3
    assert slots == [8 * BLOCK + i for i in range(4, 16)] + [4 * BLOCK, 3 * BLOCK, -1, -1]
    free, cu_b, back, status = release_ref(tables, [2, 1, 0], [33, 17, 0], [5, 4, 3, 2], 3)
    assert free == [5, 4, 3, 2] and cu_b == [0, 1, 2, 2] and back == 1 and status == 0
    assert extend_ref(t, [20, 16, 0], [13, 1, 0], [5, 4], 1, 10, 16)[-1] == 1
    assert extend_ref(t, [20, 16, 0], [29, 1, 0], [5, 4, 3, 2], 1, 10, 64)[-1] == 2
    assert extend_ref(t, [20, 16, 0], [13, 1, 0], [5, 4, 3, 2], 1, 10, 13)[-1] == 4
    assert extend_ref(t, [20, -1, 0], [13, 1, 0], [5, 4, 3, 2], 1, 10, 16)[-1] == 8
    assert release_ref(tables, [2, 1, 0], [33, 17, 0], [5, 4, 3, 2], 1)[-1] == 1
