"""The oracle of the calls for further turns, pinned by hand and by other ways to the same numbers (CPU)."""
import math

import numpy as np

from oracle import turns as T


def test_norm():
    x = np.array([[[3.0, 4.0], [0.0, 2.0]]])
    want = np.array([[[3, 4], [0, 2]]]) / np.sqrt([[[12.5], [2.0]]])
    np.testing.assert_allclose(T.norm(x), want, rtol=1e-15)
    np.testing.assert_allclose(T.norm(x, np.array([2.0, 1.0]), 0.5), x * [2, 1] / np.sqrt([[[13.0], [2.5]]]), rtol=1e-15)
    y, _ = T.norm_rope(x, [1], np.array([0.25]), None, 0.0)
    c, s = math.cos(0.25), math.sin(0.25)
    a, b = want[0, 0]
    np.testing.assert_allclose(y[0, 0], [a * c - b * s, b * c + a * s], rtol=1e-14)


def test_chunk_see():
    np.testing.assert_array_equal(T.chunk_see(2, 3), [[1, 1, 1, 1, 0], [1, 1, 1, 1, 1]])
    np.testing.assert_array_equal(T.chunk_see(3, 2, 2), [[0, 1, 1, 0, 0], [0, 0, 1, 1, 0], [0, 0, 0, 1, 1]])
    np.testing.assert_array_equal(T.chunk_see(2, 0, 1), np.eye(2))


def test_shape_logits():
    z = [1.0, -1.0, 2.0, 0.0, 4.0]
    got, _ = T.shape_logits(z, prompt=[1, 0], answer=[2, 2, 0, 9, -1], repetition=2.0, presence=0.5, frequency=0.25,
                            bias=[(3, 7.0), (3, 1.0), (8, 1.0)])
    np.testing.assert_allclose(got, [0.5 - 0.25 - 0.5, -2.0, 1.0 - 0.5 - 0.5, 1.0, 4.0])
    p, _ = T.shape_logits(z, allowed=np.array([1, 1, 0, 0, 0], bool), temperature=2.0)
    np.testing.assert_allclose(p, [1 / (1 + math.exp(-1)), 1 / (1 + math.exp(1)), 0, 0, 0], rtol=1e-14)
    np.testing.assert_array_equal(T.shape_logits([1.0, 3.0, 3.0], temperature=0)[0], [0, 1, 0])
    np.testing.assert_array_equal(T.shape_logits([1.0, 3.0], allowed=np.zeros(2, bool), temperature=1.0)[0], [0, 0])
    assert np.isnan(T.shape_logits([1.0, np.nan], temperature=1.0)[0]).all()


def test_fork_and_release():
    table = np.array([[5, 6, 7, -1], [8, -1, -1, -1], [9, 10, -1, -1]])
    # 0: 9 tokens (pages of 4), 1: 4, 2: 6
    new, lens, held, head, copies = T.page_fork(table, [9, 4, 6], [0, 0, -1], [1, 2, 3], 4, 12, head=1)
    np.testing.assert_array_equal(new, [[5, 6, 7, -1], [5, 6, 2, -1], [-1, -1, -1, -1]])
    assert list(lens) == [9, 9, 0] and list(held) == [3, 3, 0] and head == 2
    assert copies == [(-1, -1, 0), (7, 2, 1), (-1, -1, 0)]
    free, at = T.page_release(table, [3, 1, 2], new, held, [1, 2, 3], 2, 12)
    assert at == 0 and list(free) == [9, 10, 3]      # three pages, room for two: 8 is dropped
    free, at = T.page_release(table, [3, 1, 2], new, held, [0, 0, 0, 1, 2], 4, 12)
    assert at == 1 and list(free) == [0, 8, 9, 10, 2]
    # shortened inside the page that it has started, to an earlier page, to a full page, and longer than it is
    for keep, want, copied in ((8, [5, 6], 0), (6, [5, 3], 1), (4, [5], 0), (40, [5, 6, 7], 0)):
        new, lens, held, head, copies = T.page_fork(table, [9, 4, 6], [0, 1, 2], [3], 4, 12, keep=[keep, 4, 6])
        assert [p for p in new[0] if p >= 0] == want and head == copied and (copies[0] == (6, 3, 2)) == bool(copied)
