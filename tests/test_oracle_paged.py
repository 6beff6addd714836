"""Pins of the 64-bit implementations the paged cache's calls and the logits' processing are tested against."""
import numpy as np
import scipy.special

import oracle
from oracle import paged


def _pool(rng, pages, n_kv, page, d):
    return rng.standard_normal((pages, n_kv, page, d)), rng.standard_normal((pages, n_kv, page, d))


def test_paged_attention_is_dense_attention_through_the_table():
    rng = np.random.default_rng(1)
    k, v = _pool(rng, 9, 2, 4, 8)
    table, n = np.array([7, 2, 5, 0, 3]), 18
    q = rng.standard_normal((6, 8))
    out, lse, p, size = paged.paged_attend(q, k, v, table, n, 0.3)
    for h in range(6):
        K = np.concatenate([k[t, h // 3] for t in table])[:n]
        V = np.concatenate([v[t, h // 3] for t in table])[:n]
        z = 0.3 * K @ q[h]
        np.testing.assert_allclose(p[h], scipy.special.softmax(z), rtol=1e-12)
        np.testing.assert_allclose(lse[h], scipy.special.logsumexp(z), rtol=1e-12)
        ref, _, _ = oracle.dense_attend(q[h].astype(np.float32), K.astype(np.float32), V.astype(np.float32), n, 0.3)
        np.testing.assert_allclose(out[h], ref, rtol=2e-5, atol=2e-6)
        assert np.all(size[h] >= np.abs(out[h]) - 1e-12)


def test_paged_attention_without_rows_and_without_pages():
    rng = np.random.default_rng(2)
    k, v = _pool(rng, 3, 1, 4, 8)
    q = rng.standard_normal((2, 8))
    for table, n in ((np.array([0]), 0), (np.array([-1, 3]), 7)):
        out, lse, p, _ = paged.paged_attend(q, k, v, table, n, 1.0)
        assert not out.any() and np.all(lse == -np.inf) and not p.any()
    a = paged.paged_attend(q, k, v, np.array([1, -1, 2]), 12, 1.0)
    b = paged.paged_attend(q, k, v, np.array([1, 2]), 8, 1.0)
    np.testing.assert_allclose(a[0], b[0], rtol=1e-12)
    assert not a[2][:, 4:8].any()


def test_joining_two_parts_by_their_lse_is_the_whole():
    rng = np.random.default_rng(3)
    k, v = _pool(rng, 4, 1, 4, 8)
    q = rng.standard_normal((1, 8))
    whole = paged.paged_attend(q, k, v, np.array([0, 1, 2, 3]), 14, 0.5)
    x = paged.paged_attend(q, k, v, np.array([0, 1]), 8, 0.5)
    y = paged.paged_attend(q, k, v, np.array([2, 3]), 6, 0.5)
    wx, wy = np.exp(x[1] - whole[1]), np.exp(y[1] - whole[1])
    np.testing.assert_allclose(wx + wy, 1.0, rtol=1e-12)
    np.testing.assert_allclose(wx[:, None] * x[0] + wy[:, None] * y[0], whole[0], rtol=1e-11)


def test_append_is_the_tail_of_every_sequence():
    k = np.zeros((4, 1, 3, 2))
    v, pos, weight = k.copy(), np.full((4, 1, 3), -1), np.zeros((4, 1, 3))
    table = np.array([[3, 0], [1, 2]])
    new = np.arange(1.0, 11.0).reshape(5, 1, 2)
    paged.paged_append(k, v, pos, weight, table, [4, 1], [14, 1], new, -new, [0, 4, 5], np.arange(5.0)[:, None] + 1)
    assert pos[3, 0].tolist() == [10, 11, 12] and pos[0, 0].tolist() == [13, -1, -1] and pos[1, 0].tolist() == [0, -1, -1]
    assert k[0, 0, 0].tolist() == [7.0, 8.0] and v[1, 0, 0].tolist() == [-9.0, -10.0]
    assert weight[3, 0].tolist() == [1, 2, 3] and not k[2].any()


def test_eviction_by_hand():
    #      slot:  0    1    2    3    4    5    6
    weight = [1.0, 9.0, 2.0, 2.0, np.nan, 5.0, 0.5]
    pos = [0, 1, 2, 3, 4, 5, 6]
    # one sink, one recent: 0 and 6 stay; then 9 (slot 1), 5 (slot 5), then the tie at 2 to the lower position
    assert paged.evict_moves(pos, weight, 7, 4, 1, 1) == (4, [(2, 5), (3, 6)])
    assert paged.evict_moves(pos, weight, 7, 5, 1, 1) == (5, [(3, 5), (4, 6)])
    assert paged.evict_order(pos, weight, 7, 1, 1) == [0, 6, 1, 5, 2, 3, 4]
    assert paged.evict_moves(pos, weight, 7, 7, 1, 1) == (7, []) and paged.evict_moves(pos, weight, 7, -2, 1, 1) == (0, [])
    # more protected rows than places: the heavier of them
    assert paged.evict_order(pos, weight, 7, 0, 3)[:3] == [5, 6, 4]


def test_eviction_without_protection_is_the_top_m_rule():
    rng = np.random.default_rng(4)
    for _ in range(20):
        n = int(rng.integers(1, 40))
        w = rng.integers(0, 6, n).astype(np.float32)
        m = int(rng.integers(0, n + 2))
        best = np.lexsort((np.arange(n), -w.astype(np.float64)))[:m]
        stay, moves = paged.evict_moves(np.arange(n), w, n, m, 0, 0)
        held = set(range(stay)) - {t for t, _ in moves} | {s for _, s in moves}
        assert held == set(best.tolist()) and stay == min(m, n)


def test_logits_by_hand():
    y = paged.process_logits([2.0, -2.0, 4.0, 1.0, np.nan], None, 0.0, None, [0, 1, 2, 2, 9, -1], 1, 2.0, 0.5, 0.25, 2.0,
                             np.array([True, True, True, True, False]))
    # token 0 is the prompt's: halved only; 1: doubled, one time; 2: halved, two times
    np.testing.assert_allclose(y, [0.5, (-4 - 0.75) / 2, (2 - 1.0) / 2, 0.5, -np.inf])
    y = paged.process_logits([1.0, 3.0], [0.5, 4.0], 2.0, [0.0, 10.0], [], 0, 1.0, 0.0, 0.0, 1.0, None)
    np.testing.assert_allclose(y, [2.0, 11.0])
