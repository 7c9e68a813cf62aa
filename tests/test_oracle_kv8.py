"""The 8-bit cache's reference against values worked out by hand."""
import math

import numpy as np

import oracle
from oracle.kv8_oracle import E4M3


def test_e4m3_values():
    assert len(E4M3) == 127 and (np.diff(E4M3) > 0).all()
    assert E4M3[1] == 2.0 ** -9 and E4M3[8] == 2.0 ** -6 and E4M3[0x38] == 1.0 and E4M3[-1] == 448.0


def test_codes_round_to_nearest_even():
    # between 1 (0x38) and 1.125 (0x39), 1.125 and 1.25 (0x3a); below the least value
    x = [1.0, 1.0625, 1.0626, 1.1875, -1.0625, 2.0 ** -10, 3 * 2.0 ** -10, 500.0, math.inf, -math.inf, math.nan, -0.0]
    want = [0x38, 0x38, 0x39, 0x3a, 0xb8, 0x00, 0x02, 0x7e, 0x7e, 0xfe, 0x7f, 0x80]
    assert oracle.kv8_codes(x, 127).tolist() == want
    assert np.array_equal(oracle.kv8_values([0x38, 0xb9, 0x00], 130), [8.0, -9.0, 0.0])
    assert np.isnan(oracle.kv8_values([0x7f], 127)).all()


def test_exponent_is_the_least_that_holds():
    assert oracle.kv8_exponent([448.0]) == 127 and oracle.kv8_exponent([-450.0]) == 128
    assert oracle.kv8_exponent([0.0]) == 10 and oracle.kv8_exponent([3e38]) == 246
    assert oracle.kv8_exponent([math.inf, math.nan, 1.0]) == oracle.kv8_exponent([1.0]) == 119


def test_a_block_grows_to_its_largest_token():
    table, page = [[1, 0]], 16
    cache = [np.full(s, 99, np.uint8) for s in ((2, 1, 16, 128), (2, 1, 1), (2, 1, 16, 128), (2, 1, 1))]
    one, big = np.full((1, 1, 1, 128), 1.0), np.full((1, 1, 1, 128), 1.0)
    big[..., 0] = 2.0 ** 14
    oracle.kv8_append(one, one, [0], [1], table, page, cache)
    assert cache[1][1, 0, 0] == 119 and (cache[0][1, 0, 0] == 0x78).all() and (cache[0][1, 0, 1:] == 99).all()
    oracle.kv8_append(big, one, [1], [2], table, page, cache)
    # 2^14 needs 2^6; 1 is 2^-6 of it, the least normal value
    assert cache[1][1, 0, 0] == 133 and (cache[0][1, 0, 0] == 0x08).all() and cache[0][1, 0, 1, 0] == 0x78
    assert cache[3][1, 0, 0] == 119
    rows = oracle.kv8_rows(cache[0], cache[1], table[0], page, 2)
    assert (rows[0, 0] == 1.0).all() and rows[0, 1, 0] == 2.0 ** 14
    assert (cache[0][0] == 99).all()


def test_attn_weights_by_hand():
    # one kv head, two heads; two cached keys, a row that adds a third
    q = np.zeros((1, 2, 2, 128))
    q[0, 1, 0, 0], q[0, 1, 1, 0] = 1.0, 2.0
    keys = [np.zeros((1, 3, 128))]
    keys[0][0, :, 0] = [0.0, math.log(2.0), math.log(3.0)]
    lse = np.full((1, 2, 2), 5.0)
    lse[0, :, 1] = [math.log(6.0), math.log(14.0)]
    w, p, _ = oracle.kv8_attn_weights(q, lse, keys, [2], [3], [40], np.array([[[1.0, 2.0, 9.0, 9.0]]]),
                                      np.array([[[0, 1, 7, 7]]]), rows=[[1]], scale=1.0)
    assert np.allclose(w[0, 0], [1 + 1 / 6 + 1 / 14, 2 + 2 / 6 + 4 / 14, 3 / 6 + 9 / 14, 9.0])
    assert p.tolist() == [[[0, 1, 40, 7]]]
    # the first of two new rows does not see the second's key; a row without keys gives nothing
    lse[0, 1, 1] = -math.inf
    w, p, _ = oracle.kv8_attn_weights(q, lse, keys, [1], [3], [0], np.zeros((1, 1, 3)), np.zeros((1, 1, 3), int), rows=[[1, 5]],
                                      scale=1.0)
    assert np.allclose(w[0, 0], [1 / 6, 2 / 6, 0.0]) and p.tolist() == [[[0, 0, 1]]]


def test_eviction_by_hand():
    """20 tokens, 16 stay: the two newest, and those with the most weight; of equal
    ones the lowest slot; what moves keeps its value where the scales allow."""
    table, page = [[1, 0]], 16
    cache = [np.zeros(s, np.uint8) for s in ((2, 1, 16, 128), (2, 1, 1), (2, 1, 16, 128), (2, 1, 1))]
    cache[0][1, 0, :, 0] = 0x38 + np.arange(16) % 8
    cache[1][1], cache[1][0], cache[3][:] = 127, 129, 120
    cache[0][0, 0, :4, 0] = [0x40, 0x41, 0x42, 0x43]
    w = np.ones((1, 1, 24))
    w[0, 0, [3, 7, 11, 15]] = 0.5, 0.25, 0.5, 0.5
    w[0, 0, 16:] = [0.5, 0.0, 0.0, 0.75, 9, 9, 9, 9]
    p = np.arange(24)[None, None] * 2
    before = oracle.kv8_rows(cache[0], cache[1], table[0], page, 20)
    wo, po, lo = oracle.kv8_evict(w, p, [20], [40], 16, 4, table, page, cache)
    # slots 18 and 19 are protected; 3, 11, 15 and 16 tie for two places: 3 and 11 stay... 12 have weight 1
    assert lo == [16] and wo[0][7] == 0.0 and po[0][7] == 36 and po[0][15] == 38 and wo[0][15] == 0.75
    assert po[0][3] == 6 and po[0][11] == 22
    after = oracle.kv8_rows(cache[0], cache[1], table[0], page, 16)
    assert cache[1][1, 0, 0] == 129
    assert np.array_equal(after[0, [7, 15]], before[0, [18, 19]]) and np.array_equal(after[0, :7], before[0, :7])
