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


def _i32(torch, v):  # noqa: F811
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


ORDERS = {
    "sequences in turn": [(0, 0), (1, 0), (0, 1), (1, 1), (0, 2), (1, 2)],
    "descending": [(0, 6), (0, 5), (1, 3)],
    "one of them apart": [(0, 16), (0, 17), (1, 0), (0, 30)],
    "an entry twice": [(1, 4), (0, 9), (0, 9)],
    "an entry twice, apart": [(0, 9), (1, 4), (0, 9)],
    "a block again behind another": [(1, 14), (1, 15), (1, 16), (1, 13)],
}


@pytest.mark.parametrize("order", list(ORDERS))
@pytest.mark.parametrize("T", [0, 3000])
def test_an_order_that_is_not_kept_raises_the_flag(torch, order, T):  # noqa: F811
    # (T more tokens of a third sequence: 16 a wave)
    s = _cache(torch, [20, 20, 0], 1, 64, 16, [30, 30, 3010], n_positions=3010)
    where = [(2, t) for t in range(T)]
    where = where[:T // 2] + ORDERS[order] + where[T // 2:]
    good = [x for x in where if x[0] == 2] + [(0, 20), (0, 22), (1, 20), (1, 21)]
    x = torch.randn((len(where) + 4, 6 * 64), device="cuda").to(torch.bfloat16)

    def append(w):
        seqs, index = (_i32(torch, v) for v in zip(*w))
        s.cache.append(x[:len(w)], *s.dev, seqs, index, index, s.table, s.lens, torch.empty_like(x[:len(w), :256]))
        return s.cache.device_error()

    # as often as one likes: whatever other calls left behind is not taken for another owner
    for _ in range(3):
        assert append(good) == 0
        assert append(where) == 1
        assert append(good[::-1][:4][::-1]) == 0
        assert append(where[::-1][:1]) == 0
    s.cache.close()


def test_calls_of_every_kind_in_turn_raise_no_flag(torch):  # noqa: F811
    # attention's shares, and other owners of the same blocks, lie where owners look for each other
    rng = np.random.default_rng(1)
    s = _cache(torch, [300, 100, 50, 0], 2, 128, 16, [100, 300, 900, 1000], hq=8, n_positions=1100)
    q = torch.randn((40, 8 * 128), device="cuda").to(torch.bfloat16)
    for step in range(60):
        runs = [(int(b), int(rng.integers(0, 300)), int(rng.integers(1, 40))) for b in rng.permutation(4)[:rng.integers(1, 5)]]
        seqs = sum(([b] * n for b, _, n in runs), [])
        index = sum((list(range(i, i + n)) for _, i, n in runs), [])
        qkv = torch.randn((len(seqs), 12 * 128), device="cuda").to(torch.bfloat16)
        s.cache.append(qkv, *s.dev, _i32(torch, seqs), _i32(torch, index), _i32(torch, index), s.table, s.lens, qkv[:, :1024])
        if step % 2:
            s.cache.attend_prompt(q, _i32(torch, [0, 10, 20, 30, 40]), s.table, s.lens.clamp(min=10), torch.empty_like(q))
        if step % 3 == 0:
            s.cache.attend(q[:4], s.table, s.lens, torch.empty_like(q[:4]))
        assert s.cache.device_error() == 0, step
    s.cache.close()


def test_replays_raise_no_flag(torch):  # noqa: F811
    s = _cache(torch, [20, 20, 0], 1, 64, 16, [300, 300, 300])
    T = 48
    seqs, index = _i32(torch, [0] * T), _i32(torch, [0] * T)
    x, q = torch.randn((T, 6 * 64), device="cuda").to(torch.bfloat16), torch.empty((T, 256), dtype=torch.bfloat16, device="cuda")
    good = [([0] * 20 + [1] * 20 + [2] * 8, list(range(20)) + list(range(30, 50)) + list(range(8))),
            ([1] * 10 + [-1] * 10 + [0] * 28, list(range(30, 40)) + [0] * 10 + list(range(28))),
            ([2] * 30 + [0] * 10 + [1] * 8, list(range(30)) + list(range(10)) + list(range(40, 48)))]
    bad = ([0, 1] * 24, [k // 2 for k in range(48)])
    seqs.copy_(_i32(torch, good[0][0])), index.copy_(_i32(torch, good[0][1]))
    s.cache.append(x, *s.dev, seqs, index, index, s.table, s.lens, q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.cache.append(x, *s.dev, seqs, index, index, s.table, s.lens, q)
    for turn in range(4):
        for k, (b, i) in enumerate(good + [bad]):
            seqs.copy_(_i32(torch, b)), index.copy_(_i32(torch, i))
            for _ in range(2):
                g.replay()
                assert s.cache.device_error() == (k == 3), (turn, k)
    del g
    s.cache.close()
