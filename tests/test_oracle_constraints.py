"""Pins of the constraint oracle by hand-worked rows."""
import numpy as np

from oracle import constraints as oc


def test_each_rule_by_hand():
    z = [1.0, -2.0, 3.0, 4.0]
    got = oc.constrain(z, [0, 1, 2, 0], np.array([True, False, False, False]), [2], r=2.0, f=0.5, p=0.25,
                       bias=[(3, 1.0), (3, 0.5), (9, 7.0)])
    # 0: prompt only; 1: once; 2: three times with the row's own token; 3: not seen, two biases
    np.testing.assert_array_equal(got, [0.5, -4.0 - 0.5 - 0.25, 1.5 - 1.5 - 0.25, 5.5])
    got = oc.constrain([np.nan, 1.0, np.inf, 2.0], [0] * 4, np.zeros(4, bool), [], allowed=np.array([False, True, False, True]))
    np.testing.assert_array_equal(got, [-np.inf, 1.0, -np.inf, 2.0])


def test_greedy_ties_masks_and_nan():
    assert oc.greedy(np.array([1.0, 3.0, 3.0])) == 1
    assert oc.greedy(np.array([np.nan, -np.inf, -np.inf])) == 1
    assert oc.greedy(np.array([5.0, -np.inf, -np.inf]), np.array([False, True, True])) == 1
    assert oc.greedy(np.array([5.0, 1.0]), np.array([False, False])) == -1
    assert oc.greedy(np.array([np.nan, 1.0]), np.array([True, False])) == -1


def test_rows_of_chains_and_trees():
    assert oc.row_tokens(7, [8, 9], None, 2) == [7, 8, 9]
    assert oc.row_tokens(7, [8, 9, 10], [0, 0, 2], 3) == [7, 9, 10]


def test_counts():
    t = np.full((2, 5), 0x1234, np.uint16)
    oc.begin(t, 1, [4, 4, 0, 7])
    np.testing.assert_array_equal(t, [[0x1234] * 5, [0x8000, 0, 0, 0, 0x8000]])
    oc.add(t, 1, [4, 1, 4, -1, 5])
    np.testing.assert_array_equal(t[1], [0x8000, 1, 0, 0, 0x8002])
    t[1, 1] = 0x7FFF
    oc.add(t, 1, [1])
    assert t[1, 1] == 0x7FFF
