"""The float64 oracle of the cache calls over many rows, against plain loops."""
import math

import numpy as np
import pytest

from oracle import kv as okv


def _brute(q, k, v, scale, p, window, sinks):
    see = [j for j in range(p + 1) if not window or j > p - window or j < sinks]
    s = [scale * sum(a * b for a, b in zip(q, k[j])) for j in see]
    if not s:
        return [0.0] * len(v[0]), -math.inf
    top = max(s)
    e = [math.exp(x - top) for x in s]
    return [sum(x * v[j][i] for x, j in zip(e, see)) / sum(e) for i in range(len(v[0]))], top + math.log(sum(e))


@pytest.mark.parametrize("n,new", [(1, 1), (7, 7), (9, 3), (12, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 3), (3, 0), (3, 2), (1, 1), (100, 5), (2, 50)])
def test_rows_that_see_a_window_and_sinks(n, new, window, sinks):
    rng = np.random.default_rng(n * 10 + window)
    q, k, v = rng.standard_normal((new, 4, 3)), rng.standard_normal((2, n, 3)), rng.standard_normal((2, n, 3))
    out, lse, mag = okv.attend_rows(q, k, v, 0.7, okv.sees(n, new, window, sinks))
    for t in range(new):
        for h in range(4):
            o, z = _brute(q[t, h], k[h // 2], v[h // 2], 0.7, n - new + t, window, sinks)
            assert np.allclose(out[t, h], o, atol=1e-12) and abs(lse[t, h] - z) < 1e-12
    assert (mag >= np.abs(out) - 1e-12).all()


def test_a_single_row_is_the_one_token_form():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((1, 4, 8)), rng.standard_normal((2, 20, 8)), rng.standard_normal((2, 20, 8))
    out, lse, _ = okv.attend_rows(q, k, v, 0.3, okv.sees(20, 1, 6))
    ref, rlse, _ = okv.attend(q[0], k, v, 0.3, 14)
    assert np.allclose(out[0], ref) and np.allclose(lse[0], rlse)


def test_norm():
    x = np.array([[3.0, -4.0], [0.0, 0.0]])
    y = okv.head_norm(x, [2.0, 1.0], 0.0 + 1e-30)
    assert np.allclose(y[0], [6 / math.sqrt(12.5), -4 / math.sqrt(12.5)]) and (y[1] == 0).all()


def test_blocks_of_integers():
    q, s = np.zeros((32, 2), np.int8), np.zeros(2)
    okv.int8_blocks(q, s, [[1.0, -0.5], [0.25, 2.0]], [0, 1], np.float64)
    assert s[0] == 2 / 127 and s[1] == 0 and q[:2].tolist() == [[64, -32], [16, 127]]
    okv.int8_blocks(q, s, [[8.0, 0.0]], [2], np.float64)            # the scale grows: 64 / 4, -32 / 4, 16 / 4, 127 / 4
    assert s[0] == 8 / 127 and q[:3].tolist() == [[16, -8], [4, 32], [127, 0]]
    okv.int8_blocks(q, s, [[0.0, 0.0]], [0], np.float64)            # begins anew: what was there means nothing now
    assert s[0] == 2.0 ** -64 / 127 and q[0].tolist() == [0, 0]
    okv.int8_blocks(q, s, [[1e-3, 0.0]], [17], np.float64)
    assert s[1] == 1e-3 / 127 and q[17].tolist() == [127, 0]
