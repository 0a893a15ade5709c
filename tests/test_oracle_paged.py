"""The paged ops' oracle against hand-worked cases and closed forms (CPU)."""
import numpy as np
import pytest

from oracle import paged as P


def test_slots_by_hand():
    # pages of 4; request 0 holds 3 (page 9) and adds 3, request 1 starts with
    # 5, request 2 holds 4 (a full page 7) and adds none
    table, slots, pos, q_start, lens, free = P.kv_slots(
        [3, 0, 4], [3, 5, 0], [[9, -1, -1], [-1, -1, -1], [7, -1, -1]], [1, 2, 3, 4, 5], 5, 4, 10)
    assert table.tolist() == [[9, 5, -1], [4, 3, -1], [7, -1, -1]]
    assert slots == [39, 20, 21, 16, 17, 18, 19, 12, -1, -1]
    assert pos == [3, 4, 5, 0, 1, 2, 3, 4, 0, 0]
    assert q_start == [0, 3, 8, 8] and lens == [6, 5, 4] and free == [2, 0]


def test_slots_when_the_stack_runs_out():
    table, slots, pos, _, lens, free = P.kv_slots([0, 0], [5, 2], [[0, 0], [0, 0]], [8], 1, 4, 7)
    assert table.tolist() == [[8, -1], [-1, 0]]
    assert slots == [32, 33, 34, 35, -1, -1, -1] and pos == [0, 1, 2, 3, 4, 0, 1]
    assert lens == [5, 2] and free == [0, 2]


def test_slots_beyond_the_table():
    table, slots, _, _, lens, free = P.kv_slots([7], [3], [[1, 2]], [5, 6], 2, 4, 3)
    assert table.tolist() == [[1, 2]] and slots == [11, -1, -1] and lens == [10] and free == [2, 0]


def test_write_skips_what_is_out_of_range():
    k = np.arange(12.0).reshape(3, 2, 2)
    kc, vc = P.kv_write(k, -k, [3, -1, 4], np.zeros((2, 2, 2, 2)), np.zeros((2, 2, 2, 2)))
    assert (kc[1, 1] == k[0]).all() and kc.sum() == k[0].sum() and (vc == -kc).all()


def _cache(rows, page, order):
    """Rows [n, nk, hd] in pages taken in `order`."""
    n, nk, hd = rows.shape
    c = np.full((max(order) + 1, page, nk, hd), np.nan)
    for i in range(n):
        c[order[i // page], i % page] = rows[i]
    return c


def test_equal_keys_give_running_means():
    v = np.random.default_rng(0).standard_normal((7, 2, 3))
    kc, vc = _cache(np.ones((7, 2, 3)), 2, [5, 0, 3, 1]), _cache(v, 2, [5, 0, 3, 1])
    q = np.random.default_rng(1).standard_normal((4, 4, 3))
    out, written, spread, slack = P.attention(q, kc, vc, [[5, 0, 3, 1]], [7], [0, 4], 0.7)
    for t in range(4):
        for h in range(4):
            assert np.allclose(out[t, h], v[:4 + t, h // 2].mean(0), rtol=1e-14)
            assert np.allclose(spread[t, h], np.abs(v[:4 + t, h // 2]).mean(0), rtol=1e-14)
    assert written.all() and (slack > 0).all()
    out = P.attention(q, kc, vc, [[5, 0, 3, 1]], [7], [0, 4], 0.7, window=2)[0]
    assert np.allclose(out[3, 0], v[5:7, 0].mean(0), rtol=1e-14)


def test_two_keys_by_hand():
    kc, vc = _cache(np.array([[[1.0]], [[3.0]]]), 2, [0]), _cache(np.array([[[10.0]], [[20.0]]]), 2, [0])
    out = P.attention(np.array([[[0.5]]]), kc, vc, [[0]], [2], [0, 1], 2.0)[0]
    w = 1 / (1 + np.exp(1.0 - 3.0))      # scores 1 and 3
    assert np.allclose(out, 10 * (1 - w) + 20 * w, rtol=1e-14)


def test_rows_without_keys_and_rows_of_nobody():
    kc = np.ones((1, 4, 1, 2))
    out, written, _, _ = P.attention(np.ones((5, 1, 2)), kc, kc, [[0], [3]], [1, 4], [0, 3, 4], 1.0)
    # request 0: three rows over one token: only the last sees it; request 1's
    # page is not in the pool; the last row belongs to none
    assert (out[:2] == 0).all() and (out[2] == 1).all() and (out[3] == 0).all()
    assert written.tolist() == [True] * 4 + [False]


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_hidden_places_do_not_count(bad):
    v = np.ones((3, 1, 2))
    v[2] = bad
    kc, vc = _cache(v.copy(), 4, [0]), _cache(v, 4, [0])
    out = P.attention(np.ones((2, 1, 2)), kc, vc, [[0]], [3], [0, 2], 1.0)[0]
    assert (out[0] == 1).all() and not np.isfinite(out[1]).any()
