"""Pins of the float64 definitions of the cache in four bits (CPU)."""
import math

import numpy as np

import oracle.kv as okv


def test_four_bits_by_hand():
    x = np.zeros(32)
    # largest 7: exponent 0; borders go to the even code
    x[:15] = [7.0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0001, -0.7, -2.49, 6.9, 3.49, 0.0]
    assert okv.four_bits(x)[:15].tolist() == [6.0, 0.0, 0.5, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -0.5, -2.0, 6.0, 3.0, 0.0]
    x[0] = 7.0001                             # one more power of two
    assert okv.four_bits(x)[:9].tolist() == [8.0, 0.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]


def test_four_bits_half_step_and_again():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp(rng.standard_normal((50, 1)) * 3)
    y = okv.four_bits(x)
    assert np.array_equal(okv.four_bits(y), y)          # what the cache holds is stored as itself
    e = np.max(np.abs(y).reshape(-1, 32), axis=1) / 6   # 2^e or 2/3 of it
    assert (np.abs(y - x).reshape(-1, 32) <= 1.5 * e[:, None] + 1e-12).all()


def test_four_bits_of_what_is_not_finite_and_of_the_extremes():
    x = np.zeros((4, 32))
    x[0, :3] = [np.nan, 1.0, -1.0]
    x[1, :2] = [np.inf, 1.0]
    x[2, 0] = 2.0 ** -120
    x[3, 0] = 3.38e38
    y = okv.four_bits(x)
    assert y[0, :3].tolist() == [0.0, 1.0, -1.0] and y[1, :2].tolist() == [6 * 2.0 ** 125, 0.0]
    assert y[2, 0] == 0.0 and y[3, 0] == 6 * 2.0 ** 125


def test_tables_by_hand():
    t = okv.BlockTables(6, 4, 256)
    assert t.extend([2, 0], [0, 0], [65, 10], 75, 75) == ([0, 65, 75], list(range(65)) + list(range(10)),
                                                         list(range(65)) + list(range(128, 138)))
    assert t.rows == [[2], [], [0, 1], []]
    t.release([2], [64])
    assert t.rows[2] == [0] and t.free == {1, 3, 4, 5}
    # row 1 wants five blocks of four: it and the next that needs one get none, a request that needs none runs
    s = t.extend([1, 3, 0], [0, 0, 10], [257, 1, 1], 259, 259)
    assert t.refused and s[0] == [0, 257, 258, 259]     # 257 tokens exceed the longest sequence
    t.refused = False
    t2 = okv.BlockTables(3, 4, 256)
    assert t2.extend([0, 1, 2], [0, 0, 0], [64, 129, 1], 194, 194)[2][63:66] == [63, -1, -1]
    assert t2.exhausted and t2.rows == [[0], [], [], []]


def test_attention_of_one_key_and_of_equal_keys():
    q, k, v = np.ones((1, 2, 64)), np.ones((1, 1, 64)), np.arange(64.0).reshape(1, 1, 64)
    out, size, top = okv.attend(q, k, v, 0, 0.5)
    assert np.allclose(out[0, 0], np.arange(64.0)) and top.max() == 32.0
    out, _, _ = okv.attend(np.ones((1, 1, 64)), np.ones((4, 1, 64)), np.arange(256.0).reshape(4, 1, 64), 3, 0.5)
    assert np.allclose(out[0, 0], np.arange(64.0) + 96)


def test_rotation_keeps_lengths_and_turns_by_the_angle():
    x = np.zeros((2, 1, 4))
    x[:, 0, 0] = 1.0
    f = np.array([math.pi / 2, 0.1], dtype=np.float32)
    y = okv.norm_rotate(x, None, 0.0, np.array([1, 2]), f)
    assert np.allclose(y[0, 0], [0, 0, 1, 0], atol=1e-6) and np.allclose(y[1, 0], [-1, 0, 0, 0], atol=1e-6)
    y = okv.norm_rotate(x, None, 0.0, np.array([1, 2]), f, neighbours=True)
    assert np.allclose(y[0, 0], [0, 1, 0, 0], atol=1e-6)
