"""The CPU reference of the 4-bit cache against values worked out by hand and
against its own definition on random rows."""
import math

import numpy as np
import pytest

import oracle


def _row(values):
    x = np.zeros(32)
    x[:len(values)] = values
    return x[None]


@pytest.mark.parametrize("amax, e", [
    (6.0, 127), (6.96875, 127), (7.0, 128), (8.0, 128), (3.5, 127), (3.484375, 126), (1.0, 125), (0.0, 1),
    (2.0 ** -126, 1), (2.0 ** -133, 1), (float.fromhex("0x1.fep127"), 252), (math.inf, 252)])
def test_scale(amax, e):
    code, scale = oracle.kv4_quantise(_row([amax]))
    assert scale[0, 0] == e
    assert amax == 0 or amax < 7 * 2.0 ** (e - 127) or e == 252
    assert e == 1 or amax >= 7 * 2.0 ** (e - 128)


def test_codes_nearest_ties_to_even():
    # 6.5 sets X = 1; halfway values go to the even code
    x = [6.5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 0.2421875, 0.2578125, 5.03125, -0.0]
    code, _ = oracle.kv4_quantise(_row(x))
    assert code[0, :len(x)].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 14, 0, 1, 7, 8]


def test_round_trip_error():
    rng = np.random.default_rng(3)
    bits = (rng.standard_normal((500, 128)) * np.exp2(rng.integers(-20, 20, (500, 1)))).astype(np.float32)
    x = (bits.view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)
    code, e = oracle.kv4_quantise(x)
    v = oracle.kv4_values(oracle.kv4_pack(code), e)
    X = np.repeat(np.exp2(e.astype(np.float64) - 127), 32, -1)
    assert (np.abs(v - x) <= X).all()                                # amax in [6 X, 7 X) and the top step
    small = np.abs(x) < 2 * X
    assert (np.abs(v - x)[small] <= 0.25 * X[small]).all()
    again, e2 = oracle.kv4_quantise(v)                               # values of the grid stay, if the scale does
    same = np.repeat(e2 == e, 32, -1)
    assert (oracle.kv4_values(oracle.kv4_pack(again), e2) == v)[same].all() and same.mean() > 0.9


def test_page_map_by_hand():
    table = [[4, -1, -1], [2, 5, -1], [-1, -1, -1]]
    free = [0, 1, 3, -1, -1, -1]
    # b0 grows by a page, b1 ends, b2 enters with two pages
    t, f, n, slots, ok = oracle.kv4_page_map([16, 20, 0], [17, 0, 20], 16, table, free, 3, 4)
    assert f[:5] == [0, 1, 3, 2, 5] and n == 2 and ok == [1, 1, 1]
    assert t[0] == [4, 5, -1] and t[2][:2] == [2, 3]
    assert slots[0] == [5 * 16, -1, -1, -1] and slots[2] == [32, 33, 34, 35] and slots[1] == [-1] * 4
    # too few pages: b0 is served, b2 is not, a sequence that needs none is
    t, f, n, slots, ok = oracle.kv4_page_map([16, 20, 0], [17, 21, 33], 16, table, [1, 3, 0, -1, -1, -1], 2, 2)
    assert ok == [1, 1, 0] and n == 1 and slots == [[48, -1], [5 * 16 + 4, -1], [-1, -1]]


def test_verify_matches_plain_softmax():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((1, 2, 2, 8)), rng.standard_normal((1, 1, 5, 8)), rng.standard_normal((1, 1, 5, 8))
    kt, vt = rng.standard_normal((1, 2, 1, 8)), rng.standard_normal((1, 2, 1, 8))
    sees = np.array([[[True, False], [True, True]]])
    out, lse, spread, _ = oracle.kv4_verify(q, k, v, [3], [2], kt, vt, sees)
    kk, vv = np.concatenate((k[0, 0, :3], kt[0, :, 0])), np.concatenate((v[0, 0, :3], vt[0, :, 0]))
    z = kk @ q[0, 1, 1] / math.sqrt(8)
    p = np.exp(z) / np.exp(z).sum()
    assert np.allclose(out[0, 1, 1], p @ vv) and math.isclose(lse[0, 1, 1], math.log(np.exp(z).sum()))
    assert (spread >= np.abs(out) - 1e-12).all()
    out, lse, _, _ = oracle.kv4_verify(q, k, v, [0], [1])
    assert (out == 0).all() and lse[0, 0, 0] == -math.inf
