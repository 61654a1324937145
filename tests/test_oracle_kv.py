"""CPU pins of the key-value cache oracle."""
import numpy as np
import pytest
import torch

from oracle import kv


def test_e4m3_against_torch():
    v = kv.e4m3_values()
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, t, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).standard_normal(4000) * 2.0 ** np.arange(-12, 8).repeat(200),
                        (v[:126] + v[1:127]) / 2, -(v[:126] + v[1:127]) / 2, [448, 1e9, -1e9, 0.0]]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv.e4m3_encode(x), want)
    assert kv.e4m3_encode([np.nan])[0] == 0x7F


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product_and_depends_on_distance_only(interleaved):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 16))
    f = 10.0 ** -np.arange(8)

    def at(x, p):
        return kv.rotate(x, np.cos(p * f), np.sin(p * f), interleaved)

    z = (q[0::2] + 1j * q[1::2]) if interleaved else (q[:8] + 1j * q[8:])
    y = at(q, 5)
    w = (y[0::2] + 1j * y[1::2]) if interleaved else (y[:8] + 1j * y[8:])
    assert np.allclose(w, z * np.exp(5j * f), atol=1e-13)
    assert abs(at(q, 9) @ at(k, 4) - at(q, 17) @ at(k, 12)) < 1e-12


def test_attend_brute_force():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((6, 4)), rng.standard_normal((2, 5, 4)), rng.standard_normal((2, 5, 4))
    for start in (0, 2, 5):
        out, lse, share = kv.attend(q, k, v, 0.7, start)
        for h in range(6):
            e = [np.exp(0.7 * sum(q[h][i] * k[h // 3][j][i] for i in range(4))) for j in range(start, 5)]
            if not e:
                assert lse[h] == -np.inf and not out[h].any()
                continue
            assert abs(lse[h] - np.log(sum(e))) < 1e-12
            assert np.allclose(out[h], sum(x * v[h // 3][start + j] for j, x in enumerate(e)) / sum(e), atol=1e-12)
        assert np.allclose(share[:, start:].sum(1), 3 if start < 5 else 0) and not share[:, :start].any()


def test_evict_plan():
    w = np.array([0.5, 0.1, 0.1, 0.9, 0.1, 0.1], np.float32)
    p = np.arange(6)
    assert kv.evict_plan(w, p, 6, 2) == ([], [])
    # 0.9, 0.5 and the lowest of the ties stay
    assert kv.evict_plan(w, p, 3, 0) == ([2], [3])
    # positions 4 and 5 are protected, then 0.9
    assert kv.evict_plan(w, p, 3, 2) == ([0, 1, 2], [3, 4, 5])
    # by position, not by place
    assert kv.evict_plan(w, p[::-1].copy(), 3, 2) == ([2], [3])
    assert kv.evict_plan(np.array([np.nan, 0.0, -1.0], np.float32), p[:3], 1, 0) == ([0], [1])
