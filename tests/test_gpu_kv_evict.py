"""Eviction by accumulated attention weight, exactly as the oracle's plan."""
import numpy as np
import pytest

from oracle import kv as okv
from workloads.kv import DrawnCache, host_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _set(dc, b, weight=None, pos=None):
    for plain, pages, x in ((dc.weight, dc.W, weight), (dc.pos, dc.P, pos)):
        if x is not None:
            plain[b] = np.asarray(x, plain[b].dtype).reshape(plain[b].shape)
            dc.put(pages, b, plain[b])


def _check(torch, dc, budget, recent, check_lens=None):
    cache, table, lens = dc.device()
    cache.evict(table, lens, budget, recent)
    torch.cuda.synchronize()
    K, V, W, P = dc.K.copy(), dc.V.copy(), dc.W.copy(), dc.P.copy()
    got = [host_bits(cache.k), host_bits(cache.v), cache.weight.cpu().numpy(), cache.pos.cpu().numpy()]
    free = np.zeros(W.shape, bool)            # places from the budget on: what they hold afterwards is nobody's
    for b, n in enumerate(dc.lens):
        for h in range(dc.hkv):
            places, sources = okv.evict_plan(dc.weight[b][h], dc.pos[b][h], budget, recent)
            if places:
                to = dc.table[b, np.array(places) // dc.ps], h, np.array(places) % dc.ps
                of = dc.table[b, np.array(sources) // dc.ps], h, np.array(sources) % dc.ps
                for x in (K, V, W, P):
                    x[to] = x[of]
        if n > budget:
            i = np.arange(budget, n)
            free[dc.table[b, i // dc.ps], :, i % dc.ps] = True
    assert np.array_equal(lens.cpu().numpy(), np.minimum(dc.lens, budget))
    for name, x, y in zip("KVWP", got, (K, V, W, P)):
        assert np.array_equal(x[~free], y[~free], equal_nan=x.dtype.kind == "f"), name
    # a sequence within its budget is left alone, however often
    again = [x.clone() for x in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.pos, lens)]
    cache.evict(table, lens, budget, recent)
    torch.cuda.synchronize()
    for x, y in zip((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.pos, lens), again):
        assert torch.equal(x, y)
    assert cache.device_error() == 0
    cache.close()


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (64, True), (128, True)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (16, 4), (63, 63), (64, 0), (100, 31), (1000, 10)])
def test_budgets(torch, d, fp8, page, budget, recent):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 100, 101, 128, 300, 1000, 1025]
    dc = DrawnCache(lens, 2, d, page, seed=budget + recent + d, fp8=fp8)
    _check(torch, dc, budget, recent)


@pytest.mark.parametrize("n,budget", [(5000, 4999), (5000, 1), (4097, 2048), (9000, 1024), (40000, 3000), (40000, 39999),
                                      (70000, 35001)])
def test_long_sequences(torch, n, budget):
    dc = DrawnCache([n, 30, n // 2 + 1], 1, 64, 64, seed=n)
    rng = np.random.default_rng(n)
    _set(dc, 0, pos=rng.permutation(2 * n)[:n])        # out of order, as earlier evictions leave it
    _check(torch, dc, budget, min(budget, 777))


@pytest.mark.parametrize("seed", range(4))
def test_ties_zeros_infinities_and_nan(torch, seed):
    n, rng = 700, np.random.default_rng(seed)
    dc = DrawnCache([n] * 6, 2, 64, 16, seed=seed)
    _set(dc, 0, weight=np.zeros((2, n)))                                          # all the same
    _set(dc, 1, weight=rng.choice([0.0, -0.0, 1.0], (2, n)))                      # the two zeros are equal
    _set(dc, 2, weight=rng.choice([np.inf, -np.inf, np.nan, 0.5, -0.5, 1e-45], (2, n)))
    _set(dc, 3, weight=np.where(rng.random((2, n)) < 0.5, np.nan, rng.integers(0, 4, (2, n))))
    _set(dc, 4, weight=np.full((2, n), np.nan), pos=rng.permutation(n)[None].repeat(2, 0))
    _set(dc, 5, weight=np.float32(1) + np.float32(2.0 ** -23) * rng.integers(0, 5, (2, n)), pos=-rng.permutation(n)[None].repeat(2, 0))
    _check(torch, dc, 333, 50)


def test_positions_that_repeat_or_span_the_range(torch):
    n = 200
    dc = DrawnCache([n] * 4, 1, 64, 16, seed=1)
    _set(dc, 0, pos=np.full((1, n), 5))                                  # all protected: the lowest entries stay
    _set(dc, 1, pos=np.r_[np.full(n - 1, -2 ** 31), 2 ** 31 - 1])
    _set(dc, 2, pos=np.arange(n) - 2 ** 31)
    _set(dc, 3, pos=np.repeat(np.arange(n // 2), 2))
    _check(torch, dc, 60, 40)


def test_heads_keep_their_own_entries_and_pages_may_be_shared_out(torch):
    dc = DrawnCache([300, 260, 0, 301], 8, 128, 32, seed=2, spare=9)
    _check(torch, dc, 150, 20)


def test_invalid_pages_rank_last_and_raise_the_flag(torch):
    dc = DrawnCache([64, 64], 1, 64, 16, seed=3)
    cache, table, lens = dc.device()
    table[0, 2] = -9
    cache.evict(table, lens, 16, 2)
    assert cache.device_error() == 1
    # as if page 2's entries had no weight
    w, p = dc.weight[0][0].copy(), dc.pos[0][0].copy()
    w[32:48], p[32:48] = np.nan, -2 ** 31
    places, sources = okv.evict_plan(w, p, 16, 2)
    K = host_bits(cache.k)
    for to, of in zip(places, sources):
        assert np.array_equal(K[dc.table[0, to // 16], 0, to % 16], dc.K[dc.table[0, of // 16], 0, of % 16])
    assert lens.tolist() == [16, 16]
    cache.close()


def test_a_length_beyond_the_row(torch):
    dc = DrawnCache([64, 64], 1, 64, 16, seed=4, wide=0)
    cache, table, lens = dc.device()
    lens[0], lens[1] = 500, -3
    cache.evict(table, lens, 100, 2)
    assert lens.tolist() == [64, 0] and cache.device_error() == 1
    cache.close()


def test_graph_replays(torch):
    dc = DrawnCache([700, 40, 333], 2, 128, 16, seed=5)
    cache, table, lens = dc.device()
    state = [cache.k, cache.v, cache.weight, cache.pos, lens]
    start = [x.clone() for x in state]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        cache.evict(table, lens, 100, 9)
    for rep in range(3):
        runs = []
        for f in (g.replay, lambda: cache.evict(table, lens, 100, 9)):
            for x, y in zip(state, start):
                x.copy_(y)
            cache.weight.mul_(1.0 + rep)
            torch.cuda.synchronize()
            f()
            torch.cuda.synchronize()
            runs.append([x.clone().view(torch.uint8).cpu().numpy() for x in state])
        for x, y in zip(*runs):
            assert np.array_equal(x, y), rep
    cache.close()


def test_entries_beyond_four_gigabytes(torch):
    import paper_2510_23346_amd as bd
    n_pages, page, d = 90_000, 256, 128
    k = torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device="cuda")        # 5.9 GB each
    v = torch.zeros_like(k)
    cache = bd.KVCache(2, 1, d, n_pages, page, 1, k=k, v=v, weights=True)
    at = [n_pages - 1, 5, 88_000]                                                    # 600 entries in three pages
    table = torch.tensor([at], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(5)
    w = rng.permutation(768).astype(np.float32)
    for j, pg in enumerate(at):
        e = torch.arange(page, device="cuda") + j * page
        k[pg, 0] = (e % 251)[:, None].to(torch.bfloat16)
        v[pg, 0] = (e % 241)[:, None].to(torch.bfloat16)
        cache.weight[pg, 0] = torch.from_numpy(w[j * page:(j + 1) * page]).cuda()
        cache.pos[pg, 0] = e.int()
    lens = torch.tensor([600], dtype=torch.int32, device="cuda")
    cache.evict(table, lens, 300, 10)
    places, sources = okv.evict_plan(w[:600], np.arange(600), 300, 10)
    order = np.arange(600)
    order[places] = sources
    for i in range(300):
        pg, o = at[i // page], i % page
        assert float(k[pg, 0, o, 7]) == order[i] % 251 and float(v[pg, 0, o, 100]) == order[i] % 241
        assert int(cache.pos[pg, 0, o]) == order[i] and float(cache.weight[pg, 0, o]) == w[order[i]]
    assert lens.tolist() == [300] and cache.device_error() == 0
    cache.close()


@pytest.mark.parametrize("n,budget", [(8192, 4096), (8193, 4000), (28672, 9000), (28673, 20000), (8000, 7700)])
def test_lengths_where_the_keys_move_house(torch, n, budget):
    """Keys in registers, in LDS, read again; moves in LDS and in memory; one
    workgroup a head and several."""
    dc = DrawnCache([n, n - 1, 3], 2, 64, 16, seed=n + budget)
    rng = np.random.default_rng(n)
    _set(dc, 1, weight=rng.integers(0, 3, (2, n - 1)))
    _check(torch, dc, budget, 100)


def test_refusals(torch):
    import paper_2510_23346_amd as bd
    dc = DrawnCache([20, 30], 1, 64, 16, seed=6)
    cache, table, lens = dc.device()
    bare, _, _ = dc.device(weights=False)
    for f in (lambda: cache.evict(table, lens, 0), lambda: cache.evict(table, lens, 5, 6), lambda: cache.evict(table, lens, 5, -1),
              lambda: bare.evict(table, lens, 5)):
        with pytest.raises(bd.BDLoRAError) as e:
            f()
        assert e.value.code == -1
    for f in (lambda: cache.evict(table, lens[:1], 5), lambda: cache.evict(table.long(), lens, 5),
              lambda: cache.evict(table, lens.cpu(), 5)):
        with pytest.raises(ValueError):
            f()
    assert lens.tolist() == [20, 30]
    cache.evict(table[:0], lens[:0], 5)
    cache.close()
    bare.close()


@pytest.mark.parametrize("n,budget", [(24576, 9000), (24577, 9000), (36864, 12000), (36865, 9001), (70003, 66000), (70003, 200)])
def test_lengths_where_the_keys_of_long_sequences_move_house(torch, n, budget):
    dc = DrawnCache([n, n - 1, 3], 1, 64, 64, seed=n + budget)
    rng = np.random.default_rng(n)
    _set(dc, 1, weight=rng.integers(0, 3, (1, n - 1)))
    _check(torch, dc, budget, 100)


def _check_with_lost_pages(torch, dc, lost, budget, recent):
    """lost[b]: pages of sequence b (places of its table row) that the table
    names by numbers that are none.  Entries there are not there: what is left
    is ranked, as many stay as there are places for below the budget, and none
    of these is lost."""
    cache, table, lens = dc.device()
    for b, places in enumerate(lost):
        for i, j in enumerate(places):
            table[b, j] = -1 - i if i % 2 else dc.n_pages + i
    cache.evict(table, lens, budget, recent)
    torch.cuda.synchronize()
    K, V, W, P = dc.K.copy(), dc.V.copy(), dc.W.copy(), dc.P.copy()
    got = [host_bits(cache.k), host_bits(cache.v), cache.weight.cpu().numpy(), cache.pos.cpu().numpy()]
    free = np.zeros(W.shape, bool)
    moves = 0
    for b, n in enumerate(dc.lens):
        i = np.arange(n)
        there = i[~np.isin(i // dc.ps, lost[b])]
        room = int((there < budget).sum())
        for h in range(dc.hkv):
            if n <= budget:
                continue
            places, sources = okv.evict_plan(dc.weight[b][h][there], dc.pos[b][h][there], room, recent) if room else ([], [])
            to, of = (tuple((dc.table[b, there[x] // dc.ps], h, there[x] % dc.ps)) for x in
                      (np.array(places, int), np.array(sources, int)))
            moves = max(moves, len(places))
            for x in (K, V, W, P):
                x[to] = x[of]
        behind = there[there >= budget]
        free[dc.table[b, behind // dc.ps], :, behind % dc.ps] = True
    assert np.array_equal(lens.cpu().numpy(), np.minimum(dc.lens, budget))
    for name, x, y in zip("KVWP", got, (K, V, W, P)):
        assert np.array_equal(x[~free], y[~free], equal_nan=x.dtype.kind == "f"), name
    assert cache.device_error() == 1
    cache.close()
    return moves


@pytest.mark.parametrize("d,fp8", [(64, False), (128, True)])
def test_pages_lost_below_the_budget_cost_no_entry_that_stays(torch, d, fp8):
    dc = DrawnCache([400, 400, 400, 400, 399, 150], 2, d, 16, seed=d, fp8=fp8)
    rng = np.random.default_rng(3)
    _set(dc, 1, weight=rng.choice([0.0, np.nan, -np.inf, 1.0], (2, 400)))
    _set(dc, 2, weight=np.full((2, 400), np.nan))
    _set(dc, 4, pos=rng.permutation(800)[:399][None].repeat(2, 0))
    # below the budget, behind it, across it (entries 192 to 207), all below it, the last page
    lost = [[0, 3, 20], [5, 12, 13, 24], [1], list(range(13)), [2, 12, 24], []]
    assert _check_with_lost_pages(torch, dc, lost, 200, 30) > 0


@pytest.mark.parametrize("n,budget", [(12000, 6000), (20000, 10000), (30000, 11000), (50000, 20000)])
def test_pages_lost_where_the_moves_are_listed_in_memory(torch, n, budget):
    """More moves than LDS lists, keys in registers, in LDS and read again."""
    dc = DrawnCache([n, n - 1, 20, n], 1, 64, 16, seed=n)
    rng = np.random.default_rng(n)
    _set(dc, 1, weight=rng.integers(0, 3, (1, n - 1)))
    # all the weight lies behind the budget: every place below it is filled
    _set(dc, 3, weight=np.where(np.arange(n) < budget, 0.0, 1.0) + rng.random(n) / 2)
    pages = -(-n // 16)
    lost = [[0, 1, 77, budget // 16, pages - 1], sorted(rng.choice(pages, pages // 8, replace=False)), [], [0, pages - 2]]
    assert _check_with_lost_pages(torch, dc, lost, budget, 100) > 4096


def test_budgets_that_32_bits_do_not_hold_are_refused(torch):
    dc = DrawnCache([20, 30], 1, 64, 16, seed=7)
    cache, table, lens = dc.device()
    for f in (lambda: cache.evict(table, lens, 2 ** 32 + 5), lambda: cache.evict(table, lens, 5, 2 ** 32 + 1),
              lambda: cache.evict(table, lens, 2 ** 31), lambda: cache.evict(table, lens, -2 ** 32 + 5)):
        with pytest.raises(ValueError):
            f()
    assert lens.tolist() == [20, 30]
    cache.close()
