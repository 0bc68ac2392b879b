"""The float64 statements of the cache in pages (oracle/nova_paged.py) on cases small enough to be done by hand."""
import numpy as np
import pytest

from oracle import nova_paged as P


def test_pages_are_popped_from_the_top_in_order():
    table = np.full((2, 3), -1)
    table[0, 0] = 9
    t, slots, after, free, height = P.reserve(table, 16, [3, 5, 7] + [0] * 7, 3, [10, 0], [10, 0], [30, 2], 30)
    assert t.tolist() == [[9, 7, 5], [3, -1, -1]] and after == [40, 2] and height == 0
    assert slots[0, :8].tolist() == [9 * 16 + r for r in range(10, 16)] + [7 * 16, 7 * 16 + 1] and free[:3].tolist() == [3, 5, 7]


def test_slots_of_pages_that_are_none():
    t, slots, after, _, _ = P.reserve(np.array([[1, -1]]), 16, [4, 0], 1, [14], [14], [4], 4)
    assert slots[0].tolist() == [30, 31, -1, -1] and t.tolist() == [[1, 4]] and after == [18]


def test_released_pages_go_to_images_that_grow():
    t, slots, after, free, height = P.reserve(np.array([[0, 1, 2], [3, -1, -1]]), 16, [8] + [9] * 7, 1, [48, 16], [1, 16], [0, 17], 17)
    assert t.tolist() == [[0, 1, 2], [3, 2, 1]] and after == [1, 33] and height == 1 and free[:2].tolist() == [8, 9]


def test_the_first_that_asks_for_too_much_ends_it():
    table = np.array([[0, -1, -1], [1, -1, -1], [2, -1, -1]])
    t, slots, after, free, height = P.reserve(table, 16, [5, 6, 7, 7, 7, 7, 7, 7], 2, [16, 10, 16], [16, 10, 16], [1, 30, 1], 30)
    assert after == [17, 16, 16] and height == 1 and t[0].tolist() == [0, 6, -1] and t[1].tolist() == [1, -1, -1]
    assert (slots[1] >= 0).sum() == 6 and (slots[2] >= 0).sum() == 0


def test_rows_go_through_the_table():
    pool = np.arange(3 * 16 * 2, dtype=float).reshape(3, 1, 16, 2)
    rows = P.image_rows(pool, np.array([2, -1, 0]), 36)
    assert np.array_equal(rows[0, :16], pool[2, 0]) and not rows[0, 16:32].any() and np.array_equal(rows[0, 32:], pool[0, 0, :4])
    new = P.append(pool, np.full((1, 3, 1, 2), 7.0), np.array([[17, -1, 48]]))
    assert (new != pool).sum() == 2 and (new[1, 0, 1] == 7).all()


def test_what_queries_see():
    assert P.visible(5, 3, 4, True).tolist() == [3, 4, 5, 0]
    assert P.visible(2, 4, 4, True).tolist() == [0, 0, 1, 2]
    assert P.visible(5, 2, 3, False).tolist() == [5, 5, 0]


def test_attention_by_hand():
    K = [np.array([[[0.0], [np.log(3.0)], [np.nan]]])]
    V = [np.array([[[4.0], [8.0], [np.nan]]])]
    out, lse, w, reach = P.attention(np.ones((1, 2, 1, 1)), K, V, 1.0, [2], True)
    assert out[0, 0, 0, 0] == pytest.approx(7.0) and lse[0, 0, 0] == pytest.approx(np.log(4.0)) and np.isnan(out[0, 1, 0, 0])
    out, lse, _, _ = P.attention(np.ones((1, 1, 1, 1)), K, V, 1.0, [1], False, np.array([[[[0, 0, 9, -1]]]]), 1)
    assert out[0, 0, 0, 0] == 4.0 and lse[0, 0, 0] == 0.0


def test_seven_bits():
    assert P.seven_bits(np.array([127.0, 0.5, 1.5])).tolist() == [127.0, 0.0, 2.0]
    assert P.seven_bits(np.array([127.5, 3.0, 5.0])).tolist() == [128.0, 4.0, 4.0]
    assert P.seven_bits(np.array([0.25, -0.003])).tolist() == [0.25, -2.0 ** -8] and not P.seven_bits(np.zeros(3)).any()
    assert np.isnan(P.seven_bits(np.array([1.0, np.inf]))).all()


def test_select_takes_ends_ties_and_pages_of_nan():
    means = np.zeros((6, 1, 2))
    means[:, 0, 0] = [0, 5, 1, 5, 7, 0]
    table = np.arange(6)[None]
    q = np.array([[[[1.0, 0.0]]]])
    sel = lambda **kw: P.select(q, means, table, 16, [96], [1], False, **kw)[0, 0, 0].tolist()
    assert sel(first=0, recent=0, k=2) == [1, 4] and sel(first=1, recent=1, k=3) == [0, 4, 5] and sel(first=0, recent=0, k=3) == [1, 3, 4]
    assert sel(first=0, recent=0, k=8) == [0, 1, 2, 3, 4, 5, -1, -1]
    means[2] = np.nan
    assert sel(first=0, recent=0, k=2) == [2, 4]


def test_pages_of_nan_come_behind_first_and_recent_ones():
    """A page whose mean is NaN is chosen before any score, but takes no place of the `first` and `recent` ones."""
    means = np.zeros((8, 1, 2))
    means[:, 0, 0] = [0, 1, 2, 3, 4, 5, 6, 0]
    means[2:5] = np.nan
    table, q = np.arange(8)[None], np.array([[[[1.0, 0.0]]]])
    sel = lambda **kw: P.select(q, means, table, 16, [128], [1], True, **kw)[0, 0, 0].tolist()
    assert sel(first=1, recent=1, k=3) == [0, 2, 7] and sel(first=0, recent=2, k=2) == [6, 7] and sel(first=3, recent=1, k=4) == [0, 1, 2, 7]
    assert sel(first=1, recent=1, k=6) == [0, 2, 3, 4, 6, 7]


def test_the_power_of_two_is_the_one_that_holds_the_largest_number_itself():
    """127.25 is nearest to 127, and yet more than 127 ones: multiples of 2."""
    assert P.seven_bits(np.array([127.25, 3.0, -1.4])).tolist() == [128.0, 4.0, -2.0] and P.seven_bits(np.array([-127.0, 1.4])).tolist() == [-127.0, 1.0]
