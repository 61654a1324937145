"""Entry into the 8-bit cache of tokens whose entries have gaps between them, bit for
bit as in test_gpu_kv_store.py."""
import numpy as np
import pytest

from test_gpu_kv_store import Stored, torch  # noqa: F401  (torch: a fixture)
from workloads.kv import DrawnCache

pytestmark = pytest.mark.gpu


def _cache(torch, lens, hkv, d, page, room, hq=4, n_positions=300, seed=1):  # noqa: F811
    dc = DrawnCache(lens, hkv, d, page, seed=seed, int8=True, room=room)
    dc.S[np.isnan(dc.S)] = 0.0                  # (blocks whose first entry may never come)
    return Stored(torch, dc, hq, n_positions)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,page", [(4, 1, 16), (6, 3, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_runs_with_gaps(torch, d, hq, hkv, page, interleaved):  # noqa: F811
    # from a block's first entry and not, over the ends of blocks, one entry of a block, a gap
    # beside padding and other sequences; a position outside in the middle of a run
    s = _cache(torch, [0, 30, 15, 3], hkv, d, page, [90, 60, 80, 13], hq)
    runs = [(0, [0, 2, 3, 9, 15, 17, 31, 32, 33, 40, 88]), (1, [30, 33, 34, 47, 50]), (-1, [5]), (1, [65, 79]), (2, [15, 16, 18]), (3, [3, 8, 15]),
            (2, [37, 90])]
    seqs, index = (sum(x, []) for x in zip(*[([b] * len(i), i) for b, i in runs]))
    positions = [3 * t for t in range(len(seqs))]
    positions[3] = 300
    s.append(seqs, index, positions, 1, interleaved, stored=[b >= 0 and t != 3 for t, b in enumerate(seqs)])
    s.check(err=1)
    # again, larger, between what is there and over it
    runs = [(3, [4, 5, 14]), (0, [1, 3, 16, 18]), (1, [31, 35, 66])]
    seqs, index = (sum(x, []) for x in zip(*[([b] * len(i), i) for b, i in runs]))
    s.append(seqs, index, index, 2, interleaved, size=3.0)
    s.check()
    s.cache.close()


@pytest.mark.parametrize("d,hkv", [(64, 8), (128, 2)])
@pytest.mark.parametrize("keep", [0.15, 0.5, 0.97])
def test_long_runs_with_gaps(torch, d, hkv, keep):  # noqa: F811
    # (16 tokens a wave)
    rng = np.random.default_rng([d, int(100 * keep)])
    s = _cache(torch, [0, 5, 31], hkv, d, 64, [8000, 7500, 7600], hq=hkv, n_positions=8100)
    seqs, index = [], []
    for b, (start, n) in enumerate([(0, 4000), (5, 3000), (31, 3500)]):
        i = (start + np.flatnonzero(rng.random(int(n / keep) if keep > 0.4 else 2 * n) < keep)).tolist()
        seqs += [b] * len(i) + [-1]
        index += i + [0]
    for step in range(2):
        s.append(seqs, index, index, step, size=1.0 + step)
        s.check()
    s.cache.close()
