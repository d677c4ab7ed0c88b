"""Pins of the oracle's rotary positions and cache append (CPU): closed forms,
invariants and brute force."""

import math

import numpy as np
import pytest

import oracle


def test_rope_one_axis_equals_the_draft_layers_rope():
    g = np.random.default_rng(0)
    x, pos = g.standard_normal((5, 3, 8)), np.array([0, 1, 7, 100, 4095])
    got = oracle.rope_axes(x, pos[None], [4], 10000.0)
    for t in range(5):
        for h in range(3):
            for i in range(4):
                a = pos[t] * 10000.0 ** (-2 * i / 8)
                assert np.isclose(got[t, h, i], x[t, h, i] * math.cos(a) - x[t, h, i + 4] * math.sin(a), atol=1e-12)
                assert np.isclose(got[t, h, i + 4], x[t, h, i] * math.sin(a) + x[t, h, i + 4] * math.cos(a), atol=1e-12)


@pytest.mark.parametrize("per_axis", [False, True])
def test_rope_axes_frequencies(per_axis):
    # unit vectors turned by one step of one axis show that axis's frequencies only
    sections, theta = [1, 2, 3], 64.0
    for a in range(3):
        pos = np.zeros((3, 1), np.int64)
        pos[a] = 1
        ang = oracle.rope_angles(pos, sections, theta, per_axis)[0]
        first = sum(sections[:a])
        for i in range(6):
            inside = first <= i < first + sections[a]
            e = (i - first) / sections[a] if per_axis else i / 6
            assert np.isclose(float(ang[i]), theta ** -e if inside else 0.0)


def test_rope_keeps_lengths_and_inverts_and_is_its_own_gradient():
    g = np.random.default_rng(1)
    x, dy = g.standard_normal((2, 4, 2, 10))
    pos = g.integers(-50, 10 ** 6, (2, 4))
    args = (pos, [2, 2], 1e4, True)
    y = oracle.rope_axes(x, *args)
    assert np.allclose(y[..., 8:], x[..., 8:])
    assert np.allclose(y[..., :4] ** 2 + y[..., 4:8] ** 2, x[..., :4] ** 2 + x[..., 4:8] ** 2)
    assert np.allclose(oracle.rope_axes(y, *args, inverse=True), x)
    # <dy, rope(x + h e)> - <dy, rope(x)> over h, for every x_i
    dx = oracle.rope_axes(dy, *args, inverse=True)
    for i in range(x.size):
        e = np.zeros(x.size)
        e[i] = 1e-3
        num = (dy * (oracle.rope_axes(x + e.reshape(x.shape), *args) - y)).sum() / 1e-3
        assert np.isclose(num, dx.flat[i], atol=1e-9)


def test_append_then_gather_is_the_rotated_sequence():
    g = np.random.default_rng(2)
    B, Hkv, D = 3, 2, 4
    kv_len, n = np.array([20, 5, 33]), [20, 0, 17]
    start = np.concatenate([[0], np.cumsum(n)])
    T = start[-1] + 2                                  # two rows of no sequence
    q, k, v = g.standard_normal((T, 3, D)), g.standard_normal((T, Hkv, D)), g.standard_normal((T, Hkv, D))
    table = np.array([[5, 1, 0], [2, 2, 2], [3, 4, 6]])
    pool = np.full((8, Hkv, 16, D), 9.0)
    qo, kc, vc = oracle.kv_append(q, k, v, pool, pool, kv_len, start, [2], 100.0, page_table=table)
    keys, vals = oracle.gather_paged(kc, table, kv_len), oracle.gather_paged(vc, table, kv_len)
    for b in range(B):
        for j in range(n[b]):
            p, t = kv_len[b] - n[b] + j, start[b] + j
            one = oracle.rope_axes(k[t:t + 1], np.array([[p]]), [2], 100.0)[0]
            assert np.allclose(keys[b][p], one) and np.array_equal(vals[b][p], v[t])
            assert np.allclose(qo[t], oracle.rope_axes(q[t:t + 1], np.array([[p]]), [2], 100.0)[0])
        assert np.all(keys[b][:kv_len[b] - n[b]] == 9.0)
    assert np.isnan(qo[-2:]).all() and np.all(kc[[2, 7]] == 9.0)


def test_shared_prefix_equals_separate_caches():
    g = np.random.default_rng(4)
    B, k, Hq, Hkv, D, G = 5, 3, 4, 2, 8, 3
    q = g.standard_normal((B, k, Hq, D))
    kc, vc = g.standard_normal((2, B, 12, Hkv, D))
    kp, vp = g.standard_normal((2, G, 9, Hkv, D))
    kv_len, plen, start = np.array([12, 3, 7, 0, 2]), np.array([9, 4, 0]), np.array([0, 2, 2, 4])
    out, lse, spread = oracle.verify_shared(q, kc, vc, kv_len, kp, vp, plen, start, 0.3)
    for b in range(B):
        i = {0: 0, 1: 0, 2: 2, 3: 2}.get(b)           # group 1 is empty, sequence 4 in none
        n = 0 if i is None else plen[i]
        lead = [x[i, :n] if i is not None else x[0, :0] for x in (kp, vp)]
        K, V = (np.concatenate([a, c[b, :kv_len[b]]])[None] for a, c in zip(lead, (kc, vc)))
        if kv_len[b] >= k:
            ro, rl = oracle.verify_attention(q[b:b + 1], K, V, [n + kv_len[b]], 0.3)
            assert np.allclose(out[b], ro[0]) and np.allclose(lse[b], rl[0])
    # no own key visible: the prefix alone, or nothing
    assert np.all(lse[3] == -np.inf) and not out[3].any()
    assert np.all(np.isinf(lse[4, 0])) and np.all(np.isfinite(lse[4, 1:]))
    assert np.all(spread >= np.abs(out) - 1e-12)
