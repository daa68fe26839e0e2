"""The plain model of the paged cache against what it has to be: by hand, and by other means."""
from fractions import Fraction

import numpy as np
import pytest
from scipy.special import softmax

from oracle import paged_oracle as O


def test_plan_by_hand():
    table = np.array([[4, 7, -1], [2, -1, -1], [5, 1, 6]])
    got = O.plan([3, 1, -1], [30, 15, 33], [0, 3, 8, 9, -1, -1, -1, -1, -1, -1], 4, table, 16, 4)
    # request 2 gives back 5, 1, 6; request 0 needs one block (30 + 3 > 32) and takes the top, 6; request 1 fills its block
    assert got["new_seq_len"].tolist() == [33, 16, 0]
    assert got["free_list"].tolist()[:7] == [0, 3, 8, 9, 5, 1, 6]
    assert got["new_free_count"].tolist() == [6]
    assert got["block_table"].tolist() == [[4, 7, 6], [2, -1, -1], [5, 1, 6]]
    assert got["slot_map"].tolist() == [7 * 16 + 14, 7 * 16 + 15, 6 * 16, 2 * 16 + 15]
    assert got["tok_start"].tolist() == [0, 3, 4, 4] and got["tok_len"].tolist() == [3, 1, 0] and not got["refused"]


def test_plan_refuses_in_order():
    table = np.full((4, 2), -1)
    got = O.plan([17, 20, 1, 33], [0, 0, 0, 0], [3, 1, 2, -1], 3, table, 16, 100)
    # the second asks for two where one is left, and so the third gets none either; the fourth is longer than its table
    assert got["tok_len"].tolist() == [17, 0, 0, 0] and got["refused"]
    assert got["new_free_count"].tolist() == [1]
    assert (got["slot_map"][17:] == -1).all()
    assert O.plan([5, 5], [0, 0], [0, 1], 2, np.full((2, 1), -1), 16, 9)["tok_len"].tolist() == [5, 0]


@pytest.mark.parametrize("seed", range(20))
def test_blocks_are_neither_lost_nor_held_twice(seed):
    rng = np.random.default_rng(seed)
    seqs, width, block, n_blocks = 6, 5, 16, 17
    table, length = np.full((seqs, width), -1), np.zeros(seqs, int)
    free, count = np.arange(n_blocks), n_blocks
    for _ in range(40):
        got = O.plan(rng.integers(-1, 30, seqs), length, free, count, table, block, int(rng.integers(0, 120)))
        table, length, free, count = got["block_table"], got["new_seq_len"], got["free_list"], int(got["new_free_count"][0])
        held = [int(table[b, j]) for b in range(seqs) for j in range(-(-length[b] // block))]
        assert sorted(held + [int(x) for x in free[:count]]) == list(range(n_blocks))


def test_codes_are_the_nearest_ones():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((13, 1, 64)).astype(np.float32)
    cache = O.Cache(2, 1, 16, 64)
    cache.append(x[:5], [16, 17, 18, 19, 20])
    first = cache.scale[1, 0]
    assert first == np.float32(np.abs(x[:5]).max() / 127)
    cache.append(x[5:], range(21, 29))
    s = cache.scale[1, 0]
    assert s >= first and (cache.codes[0] == 0).all()
    exact = np.array([[Fraction(float(v)) / Fraction(float(s)) for v in row] for row in x[:, 0]])
    off = np.abs((cache.codes[1, 0, :13] - exact).astype(float))
    assert off[5:].max() <= 0.5 and off[:5].max() <= 0.5 + 0.5 * float(first / s) + 1e-12


def test_ties_floor_and_what_is_not_finite():
    cache = O.Cache(1, 4, 16, 64)
    x = np.zeros((2, 4, 64))
    x[0, 0, :4] = [127.0, 0.5, 1.5, -2.5]
    x[0, 1, 0] = 2.0 ** -41
    x[0, 2, 0], x[0, 3, 1] = np.inf, np.nan
    cache.append(x[:1], [0])
    assert cache.codes[0, 0, 0, :4].tolist() == [127, 0, 2, -2]
    assert cache.scale[0, 1] == 2.0 ** -40 and cache.codes[0, 1, 0, 0] == 0        # a tie with zero
    assert np.isnan(cache.scale[0, 2:]).all() and (cache.codes[0, 2:] == 0).all()
    cache.append(x[1:], [1])
    assert np.isnan(cache.scale[0, 2:]).all()
    cache.append(x[1:], [0])
    assert cache.scale[0].tolist() == [2.0 ** -40] * 4


def test_v_bytes_are_where_the_layout_puts_them():
    rng = np.random.default_rng(2)
    for block, dim in ((16, 64), (64, 128)):
        cache = O.Cache(2, 3, block, dim)
        cache.codes = rng.integers(-127, 128, cache.codes.shape)
        data = cache.bytes(True)
        for _ in range(200):
            n, h, r, d = (int(rng.integers(0, m)) for m in cache.codes.shape)
            place = r // 16 * 16 * dim + d // 64 * 1024 + r // 4 % 4 * 256 + d % 16 * 16 + d // 16 % 4 * 4 + r % 4
            assert int(data[n, h, place]) - 128 == cache.codes[n, h, r, d]
        for layout in (False, True):
            again = O.Cache.from_bytes(cache.bytes(layout), cache.scale, block, dim, layout)
            assert (again.codes == cache.codes).all()


def test_attention_against_a_library_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 6, 64)), rng.standard_normal((2, 9, 64)), rng.standard_normal((2, 9, 64))
    there = np.ones(9, bool)
    there[4] = False
    out, _, _, _ = O.attention(q, k, v, there, 0.3, [0, 4, 9])
    assert (out[0] == 0).all()
    for r, keep in ((1, [0, 1, 2, 3]), (2, [0, 1, 2, 3, 5, 6, 7, 8])):
        for h in range(6):
            p = softmax(k[h // 3][keep] @ q[r, h] * 0.3)
            np.testing.assert_allclose(out[r, h], p @ v[h // 3][keep], rtol=1e-12, atol=1e-14)
