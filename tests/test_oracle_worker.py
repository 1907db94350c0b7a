"""The oracle of a worker's step against cases worked by hand."""
import numpy as np
import pytest

from oracle import worker as ow


def _off(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)


def test_groups_by_hand():
    chains = [[1, 2, 3, 4], [9], [1, 2, 7], [1, 2, 3, 5, 6], [8, 8], [9], []]
    flat, off = np.concatenate([np.array(c, np.uint64) for c in chains]), _off([len(c) for c in chains])
    order, goff, shared, n = ow.prefix_groups(flat, off, 2)
    assert order.tolist() == [0, 2, 3, 1, 4, 5, 6] and n == 5
    assert goff.tolist() == [0, 3, 4, 5, 6, 7, 7, 7]
    assert shared.tolist() == [2, 0, 0, 0, 0, 0, 0]
    order, goff, shared, n = ow.prefix_groups(flat, off, 1)
    assert order.tolist() == [0, 2, 3, 1, 5, 4, 6] and n == 4
    assert shared.tolist() == [2, 1, 0, 0, 0, 0, 0]


def test_groups_missing_hashes_by_hand():
    chains = [[1, 2, 0, 0], [1, 5, 0, 0], [1, 2, 0, 0, 0], [7, 8, 0], [7, 8, 0]]
    flat, off = np.concatenate([np.array(c, np.uint64) for c in chains]), _off([len(c) for c in chains])
    order, goff, shared, n = ow.prefix_groups(flat, off, 1)
    assert order.tolist() == [0, 1, 2, 3, 4] and n == 2 and shared[:2].tolist() == [1, 2]
    order, goff, shared, n = ow.prefix_groups(flat, off, 2)
    assert order.tolist() == [0, 2, 1, 3, 4] and n == 3 and shared[:3].tolist() == [2, 0, 2]
    assert ow.prefix_groups(flat, off, 3)[3] == 5


def test_tables_by_hand():
    # request 0 holds blocks 50, 51 and gets one more token; 1 and 2 are new and share 2 blocks
    tables = np.full((3, 4), -1, np.int32)
    tables[0, :2] = 50, 51
    t, slots, q_off, taken = ow.block_tables(tables, [33, 40, 36], [1, 40, 4], [2, 0, 0], [7, 8, 9, 10, 11, 12], 50,
                                             np.array([0, 1, 3, 3]), [0, 2, 0])
    assert t.tolist() == [[50, 51, 7, -1], [8, 9, 10, -1], [8, 9, 11, -1]] and taken == 5
    assert q_off.tolist() == [0, 1, 41, 45]
    assert slots[0] == 16 * 7 and slots[1:17].tolist() == list(range(128, 144))
    assert slots[40] == 16 * 10 + 7 and slots[41:45].tolist() == [176, 177, 178, 179] and (slots[45:] == -1).all()
    # the second of the group brings the prefix too: its tokens there are the first one's to write
    _, slots, _, _ = ow.block_tables(tables, [33, 40, 36], [1, 40, 36], [2, 0, 0], [7, 8, 9, 10, 11, 12], 90,
                                     np.array([0, 1, 3, 3]), [0, 2, 0])
    assert (slots[41:73] == -1).all() and slots[73] == 176


def test_attention_by_hand():
    # equal scores: the mean of the values seen; a key that is not seen may hold anything
    k, v = np.zeros((2, 16, 1, 8)), np.zeros((2, 16, 1, 8))
    v[1, :3, 0, 0] = 1, 3, 8
    k[1, 3:], v[1, 3:], v[1, 2, 0, 1] = np.nan, np.inf, np.nan
    out, lse, mean, most = ow.attention(np.ones((2, 2, 8)), k, v, np.array([[1]]), [3], [0, 2])
    assert np.allclose(out[0, :, 0], 2) and np.allclose(out[1, :, 0], 4)
    assert (out[0, :, 1] == 0).all() and np.isnan(out[1, :, 1]).all()
    assert np.allclose(lse, np.log([[2, 2], [3, 3]]))
    out, lse, _, _ = ow.attention(np.ones((1, 1, 8)), k, v, np.array([[-1]]), [3], [0, 1])
    assert (out == 0).all() and (lse == -np.inf).all()


@pytest.mark.parametrize("seed", range(3))
def test_attention_both_ways(seed):
    """The matrix form and the row by row form (taken for values that are not finite) agree."""
    rng = np.random.default_rng(seed)
    k, v = rng.normal(size=(6, 16, 2, 16)), rng.normal(size=(6, 16, 2, 16))
    tables, kv, q_off = np.array([[0, 3], [5, 2]]), [19, 32], np.array([0, 4, 9])
    q = rng.normal(size=(9, 6, 16))
    a = ow.attention(q, k, v, tables, kv, q_off)
    k2, v2 = k.copy(), v.copy()
    k2[3, 5:], v2[3, 5:] = np.nan, np.nan      # behind request 0's last token: taken away with its rows
    k2[2, 15], v2[2, 15] = np.inf, np.nan      # request 1's last token
    b = ow.attention(q, k2, v2, tables, kv, q_off)
    for x, y in zip(a, b):
        assert np.allclose(x[:8], y[:8], rtol=1e-12)
    assert np.isnan(b[0][8]).all()
