"""Attention of one new token over the paged key-value cache, against the
float64 oracle.

Tolerances (per element, from the formula):
- a score is a sum of d products in fp32: off by at most es = (d + 4) 2^-24
  scale sum |q||k| (and a rounding of the result);
- a probability is then off by a factor of at most 2 es + 2^-20, and the
  kernel holds it in 16 or more bits for the sum over values: 2^-15;
- out adds one rounding to bf16 (8 significant bits: half a step is at most
  2^-8 of the result).
"""
import numpy as np
import pytest

import workloads as wl
from oracle import kv as okv
from workloads.gpu import device_to_float
from workloads.kv import DrawnCache, host_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _queries(torch, B, hq, d, seed, scale=2.0):
    bits, x = wl.bf16_round(np.random.default_rng([seed, 5]).standard_normal((B, hq * d)) * scale)
    return torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16), x.astype(np.float64).reshape(B, hq, d)


def _check(dc, q, out, lse, weight, starts, scale, B=None, old_weight=None):
    """All of a call's results against the oracle."""
    hq, d = q.shape[1], q.shape[2]
    out = device_to_float(out).astype(np.float64).reshape(-1, hq, d)
    lse = lse.cpu().numpy() if lse is not None else None
    W = weight.cpu().numpy() if weight is not None else None
    G = hq // dc.hkv
    for b in range(len(dc.lens) if B is None else B):
        n, s = int(dc.lens[b]), 0 if starts is None else max(0, int(starts[b]))
        ref, rlse, share = okv.attend(q[b], dc.k[b], dc.v[b], scale, min(s, n))
        es = np.zeros((hq, max(n, 1)))
        mag = np.zeros_like(ref)
        for h in range(hq):
            if n > s:
                es[h, :n] = (d + 4) * 2.0 ** -24 * scale * (np.abs(dc.k[b][h // G]) @ np.abs(q[b, h]))
                p = np.exp(scale * (dc.k[b][h // G][:, :] @ q[b, h]) - rlse[h])[s:]
                mag[h] = p @ np.abs(dc.v[b][h // G][s:])
        top = es.max(1)
        tol = 2.0 ** -8 * np.abs(ref) + (4 * top[:, None] + 2.0 ** -15 + 2.0 ** -20) * mag
        bad = ~(np.abs(out[b] - ref) <= tol)
        assert not bad.any(), (b, n, s, np.argwhere(bad)[:4], out[b][bad][:4], ref[bad][:4], tol[bad][:4])
        if lse is not None:
            if n <= s:
                assert (lse[b] == -np.inf).all(), (b, lse[b])
            else:
                assert (np.abs(lse[b] - rlse) <= 2 * top + 2.0 ** -20 * (1 + np.abs(rlse))).all(), (b, lse[b], rlse)
        if W is not None:
            got, old = dc.take(W, b, n), dc.weight[b] if old_weight is None else old_weight[b]
            err = (4 * top.max() + 2.0 ** -19) * share + 2.0 ** -22 * (np.abs(old) + share)
            assert (np.abs(got - old - share) <= err).all(), (b, np.abs(got - old - share).max())


def _lens_all():
    return [1, 0, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 257, 511, 700, 1023, 1500]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 2), (3, 3)])
@pytest.mark.parametrize("fp8", [False, True])
def test_lengths_pages_heads_formats(torch, d, page, hq, hkv, fp8):
    dc = DrawnCache(_lens_all(), hkv, d, page, seed=d + page + hq + fp8, fp8=fp8, k_scale=0.02 if fp8 else 1.0,
                    v_scale=0.011 if fp8 else 1.0)
    cache, table, lens = dc.device(n_q_heads=hq)
    B = len(dc.lens)
    q, qv = _queries(torch, B, hq, d, seed=page)
    out = torch.full((B, hq * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, hq), float("nan"), device="cuda")
    before = (host_bits(cache.k), host_bits(cache.v), cache.pos.cpu().numpy())
    cache.attend(q, table, lens, out, lse=lse, accumulate=True)
    _check(dc, qv, out, lse, cache.weight, None, d ** -0.5)
    # nothing else is written: other weights, keys, values and positions
    W = cache.weight.cpu().numpy()
    mine = np.zeros(W.shape, bool)
    for b in range(B):
        p, s = dc.where(b)
        mine[p, :, s] = True
    assert np.array_equal(W[~mine], dc.W[~mine], equal_nan=True)
    for x, y in zip(before, (host_bits(cache.k), host_bits(cache.v), cache.pos.cpu().numpy())):
        assert np.array_equal(x, y)
    # without weights the same out
    out2 = torch.empty_like(out)
    cache.attend(q, table, lens, out2)
    torch.cuda.synchronize()
    assert np.array_equal(W, cache.weight.cpu().numpy(), equal_nan=True)
    assert torch.equal(out.view(torch.int16), out2.view(torch.int16))
    assert cache.device_error() == 0
    cache.close()


@pytest.mark.parametrize("hq,hkv", [(16, 1), (17, 1), (40, 2), (64, 1), (32, 8), (5, 1)])
def test_group_sizes(torch, hq, hkv):
    dc = DrawnCache([200, 1, 77, 0, 130], hkv, 128, 16, seed=hq)
    cache, table, lens = dc.device(n_q_heads=hq)
    q, qv = _queries(torch, 5, hq, 128, seed=hq)
    out, lse = torch.full((5, hq * 128), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.empty(5, hq, device="cuda")
    cache.attend(q, table, lens, out, lse=lse, accumulate=True)
    _check(dc, qv, out, lse, cache.weight, None, 128 ** -0.5)
    cache.close()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("fp8", [False, True])
def test_starts_leave_rows_partly_or_wholly_masked(torch, page, fp8):
    lens = [300, 300, 300, 300, 300, 64, 64, 17, 1, 0, 1000, 1000]
    starts = [0, 1, 15, 299, 300, 63, 31, 16, 0, 0, 777, -5]
    dc = DrawnCache(lens, 2, 128, page, seed=3, fp8=fp8, k_scale=0.02 if fp8 else 1.0, v_scale=0.02 if fp8 else 1.0)
    nan = 0xFF if fp8 else 0x7FFF
    for b, s in enumerate(starts):               # entries before the start may hold anything, their pages be gone
        if s > 0:
            p, o = dc.where(b, min(s, lens[b]))
            dc.K[p, :, o], dc.V[p, :, o] = nan, nan
            gone = min(s, lens[b]) // page
            dc.table[b, :gone] = -1
    cache, table, dl = dc.device(n_q_heads=8)
    q, qv = _queries(torch, len(lens), 8, 128, seed=4)
    out = torch.full((len(lens), 8 * 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(len(lens), 8, device="cuda")
    st = torch.tensor(starts, dtype=torch.int32, device="cuda")
    old = cache.weight.clone()
    cache.attend(q, table, dl, out, starts=st, lse=lse, accumulate=True, scale=0.05)
    _check(dc, qv, out, lse, None, starts, 0.05)
    W = cache.weight.cpu().numpy()
    for b, s in enumerate(starts):
        n, s = lens[b], min(max(s, 0), lens[b])
        i = np.arange(s, n)
        _, _, share = okv.attend(qv[b], dc.k[b], dc.v[b], 0.05, s)
        p, o = dc.table[b, i // page], i % page
        got = W[p, :, o].T
        assert np.allclose(got, dc.weight[b][:, s:] + share[:, s:], rtol=1e-5, atol=1e-6), b
        W[p, :, o] = old.cpu().numpy()[p, :, o]
    assert np.array_equal(W, old.cpu().numpy(), equal_nan=True)          # nothing else was touched
    assert cache.device_error() == 0
    cache.close()


def test_a_long_sequence_beside_short_ones_and_the_same_bits_again(torch):
    lens = [70001, 3, 900, 0, 20000, 1]
    dc = DrawnCache(lens, 1, 64, 64, seed=8)
    cache, table, dl = dc.device(n_q_heads=4)
    q, qv = _queries(torch, 6, 4, 64, seed=8, scale=3.0)
    out, lse = torch.empty(6, 256, dtype=torch.bfloat16, device="cuda"), torch.empty(6, 4, device="cuda")
    cache.attend(q, table, dl, out, lse=lse, accumulate=True)
    _check(dc, qv, out, lse, cache.weight, None, 0.125)
    first = (out.clone(), lse.clone())
    for _ in range(5):
        junk = torch.randn(1 << 22, device="cuda")          # something else on the device in between
        junk.mul_(2.0)
        cache.attend(q, table, dl, out, lse=lse)
        assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])
    cache.close()


@pytest.mark.parametrize("lens", [[9001, 8013, 8490, 9100], [1100, 990, 1300, 1201, 1055, 1499]])
@pytest.mark.parametrize("hq,d", [(1, 64), (4, 128)])
def test_sequences_that_meet_within_a_workgroup(torch, lens, hq, d):
    """Each goes over many workgroups, and those at the ends have parts of
    two: both may be completed, and added, by one workgroup."""
    dc = DrawnCache(lens, 1, d, 16, seed=hq)
    cache, table, dl = dc.device(n_q_heads=hq)
    q, qv = _queries(torch, len(lens), hq, d, seed=8)
    runs = []
    for _ in range(8):
        out = torch.full((len(lens), hq * d), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((len(lens), hq), float("nan"), device="cuda")
        cache.attend(q, table, dl, out, lse=lse)
        runs.append((out, lse))
    _check(dc, qv, *runs[0], None, None, d ** -0.5)
    for out, lse in runs[1:]:
        assert torch.equal(out.view(torch.int16), runs[0][0].view(torch.int16)) and torch.equal(lse, runs[0][1])
    cache.close()


def test_large_batch_of_short_sequences(torch):
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 40, 700)
    dc = DrawnCache(lens, 1, 64, 16, seed=9)
    cache, table, dl = dc.device(n_q_heads=4, max_seqs=1000)
    q, qv = _queries(torch, 700, 4, 64, seed=9)
    out, lse = torch.full((700, 256), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.empty(700, 4, device="cuda")
    cache.attend(q, table, dl, out, lse=lse, accumulate=True)
    _check(dc, qv, out, lse, cache.weight, None, 0.125)
    cache.close()


def test_row_strides_and_a_wider_table(torch):
    dc = DrawnCache([100, 33, 260], 2, 128, 16, seed=10)
    cache, table, dl = dc.device(n_q_heads=8)
    q, qv = _queries(torch, 3, 8, 128, seed=10)
    rows = torch.full((3, 8 * 128 + 512), float("nan"), dtype=torch.bfloat16, device="cuda")
    rows[:, :1024] = q
    wide = torch.full((3, 8 * 128 + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 8:8 + 1024]
    big = torch.full((3, table.shape[1] + 9), -3, dtype=torch.int32, device="cuda")
    big[:, 4:4 + table.shape[1]] = table
    cache.attend(rows[:, :1024], big[:, 4:4 + table.shape[1]], dl, out.unflatten(1, (8, 128)))
    _check(dc, qv, out.contiguous(), None, None, None, 128 ** -0.5)
    assert (wide[:, :8] == 7).all() and (wide[:, 8 + 1024:] == 7).all()
    cache.close()


def test_infinite_and_nan_entries(torch):
    """Values of entries that are attended to follow the formula: a NaN score
    makes the row NaN, an infinite value the output infinite, scores that are
    all -infinity an empty row."""
    dc = DrawnCache([40, 40, 40, 40], 1, 64, 16, seed=12)
    one, inf = 0x3F80, 0x7F80
    dc.put(dc.K, 0, np.where(np.arange(40)[None, :, None] == 7, 0x7FC0, dc.take(dc.K, 0, 40)).astype(np.uint16))
    v1 = dc.take(dc.V, 1, 40).copy()
    v1[0, 20, 3] = inf
    dc.put(dc.V, 1, v1)
    k2 = np.full((1, 40, 64), 0, np.uint16)
    k2[0, :, 0] = inf | 0x8000
    dc.put(dc.K, 2, k2)
    k3 = dc.take(dc.K, 3, 40).copy()             # all but one entry -infinity
    k3[0, :, :] = 0
    k3[0, :, 0] = inf | 0x8000
    k3[0, 33, 0] = one
    dc.put(dc.K, 3, k3)
    cache, table, dl = dc.device(n_q_heads=2)
    q, _ = _queries(torch, 4, 2, 64, seed=12)
    q[2:] = 0
    q[2:, 0::64] = 1.0
    out, lse = torch.full((4, 128), 5.0, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 2, device="cuda")
    q[2:, 1:64], q[2:, 65:] = 0.0, 0.0
    cache.attend(q, table, dl, out, lse=lse)
    y = device_to_float(out).reshape(4, 2, 64)
    s = lse.cpu().numpy()
    assert np.isnan(y[0]).all() and np.isnan(s[0]).all()
    assert np.isposinf(y[1][:, 3]).all() and np.isfinite(np.delete(y[1], 3, 1)).all() and np.isfinite(s[1]).all()
    assert (y[2] == 0).all() and np.isneginf(s[2]).all()
    assert np.array_equal(y[3], np.broadcast_to(dc.v[3][0, 33], (2, 64))) and np.allclose(s[3], 0.125)
    cache.close()


def test_scores_far_apart(torch):
    """Scores of thousands, rising and falling along the sequence."""
    dc = DrawnCache([500, 500], 1, 128, 32, seed=13)
    cache, table, dl = dc.device(n_q_heads=4)
    q, qv = _queries(torch, 2, 4, 128, seed=13, scale=60.0)
    out, lse = torch.empty(2, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, device="cuda")
    for scale in (1.0, -1.0):
        cache.attend(q, table, dl, out, lse=lse, scale=scale)
        y, s = device_to_float(out).reshape(2, 4, 128), lse.cpu().numpy()
        for b in range(2):
            ref, rl, _ = okv.attend(qv[b], dc.k[b], dc.v[b], scale)
            assert np.allclose(s[b], rl, rtol=1e-5)
            assert np.abs(y[b] - ref).max() < 0.05      # (d + 4) 2^-24 sum |q||k| = 0.05 of the score
    cache.close()


def test_invalid_pages_and_lengths_raise_the_flag_and_are_left_out(torch):
    dc = DrawnCache([64, 64, 64, 64], 1, 64, 16, seed=14)
    cache, table, dl = dc.device(n_q_heads=2)
    q, qv = _queries(torch, 4, 2, 64, seed=14)
    out, lse = torch.empty(4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 2, device="cuda")
    table[0, 1] = dc.n_pages                  # one page of the four is no page
    table[1, :4] = -1
    narrow = table[:, :4]
    dl[2], dl[3] = 1000, -4                   # beyond the row, negative
    cache.attend(q, narrow, dl, out, lse=lse, accumulate=True)
    assert cache.device_error() == 1 and cache.device_error() == 0
    y, s = device_to_float(out).astype(np.float64).reshape(4, 2, 64), lse.cpu().numpy()
    keep = np.r_[0:16, 32:64]
    for b, (k, v) in ((0, (dc.k[0][:, keep], dc.v[0][:, keep])), (2, (dc.k[2], dc.v[2]))):
        ref, rl, _ = okv.attend(qv[b], k, v, 0.125)
        assert np.allclose(y[b], ref, rtol=2 ** -8, atol=2e-3) and np.allclose(s[b], rl, atol=1e-4)
    for b in (1, 3):
        assert (y[b] == 0).all() and np.isneginf(s[b]).all()
    cache.close()


def test_entries_beyond_four_gigabytes(torch):
    """Pages whose bytes lie past 2^32 and whose entries pass 2^24."""
    n_pages, page, d = 90_000, 256, 128
    import paper_2510_23346_amd as bd
    k = torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device="cuda")        # 5.9 GB each
    v = torch.zeros_like(k)
    dc = DrawnCache([700, 300], 1, d, page, seed=15, spare=0)
    at = torch.tensor([n_pages - 1, 0, n_pages - 3, 89_000, 66_000], device="cuda")[:dc.n_pages]
    k[at] = torch.from_numpy(dc.K.view(np.int16)).cuda().view(torch.bfloat16)
    v[at] = torch.from_numpy(dc.V.view(np.int16)).cuda().view(torch.bfloat16)
    table = torch.from_numpy(np.where((dc.table >= 0) & (dc.table < dc.n_pages), at.cpu().numpy()[np.clip(dc.table, 0, dc.n_pages - 1)],
                                      -1).astype(np.int32)).cuda()
    cache = bd.KVCache(4, 1, d, n_pages, page, 2, k=k, v=v)
    q, qv = _queries(torch, 2, 4, d, seed=15)
    out, lse = torch.empty(2, 4 * d, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 4, device="cuda")
    cache.attend(q, table, torch.from_numpy(dc.lens).cuda(), out, lse=lse)
    _check(dc, qv, out, lse, None, None, d ** -0.5)
    assert cache.device_error() == 0
    cache.close()


def test_another_stream_and_graph_replays_over_changed_lengths(torch):
    dc = DrawnCache([600, 900, 40], 2, 128, 16, seed=16)
    cache, table, dl = dc.device(n_q_heads=8)
    q, qv = _queries(torch, 3, 8, 128, seed=16)
    out, lse = torch.empty(3, 1024, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.attend(q, table, dl, out, lse=lse, stream=side)
    side.synchronize()
    _check(dc, qv, out, lse, None, None, 128 ** -0.5)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        cache.attend(q, table, dl, out, lse=lse, accumulate=True)
    eager, elsel = torch.empty_like(out), torch.empty_like(lse)
    for rep, n in enumerate(([600, 900, 40], [1, 0, 17], [599, 33, 40], [600, 900, 40])):
        dl.copy_(torch.tensor(n, dtype=torch.int32))
        cache.weight.zero_()
        g.replay()
        torch.cuda.synchronize()
        w = cache.weight.clone()
        cache.weight.zero_()
        cache.attend(q, table, dl, eager, lse=elsel, accumulate=True)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)) and torch.equal(lse, elsel), rep
        assert torch.equal(w, cache.weight), rep
        out.fill_(float("nan"))
    cache.close()


def test_refusals(torch):
    import paper_2510_23346_amd as bd
    dc = DrawnCache([20, 30], 1, 64, 16, seed=17)
    cache, table, dl = dc.device(n_q_heads=4, weights=False)
    q, _ = _queries(torch, 2, 4, 64, seed=1)
    out = torch.zeros_like(q)
    for f in (lambda: cache.attend(q.float(), table, dl, out), lambda: cache.attend(q[:, :128], table, dl, out),
              lambda: cache.attend(q, table.long(), dl, out), lambda: cache.attend(q, table[:1], dl, out),
              lambda: cache.attend(q, table, dl[:1], out), lambda: cache.attend(q, table, dl.float(), out),
              lambda: cache.attend(q, table, dl, out, starts=dl[:1]), lambda: cache.attend(q, table, dl, out[:1]),
              lambda: cache.attend(q, table, dl, out, lse=torch.zeros(2, 3, device="cuda")),
              lambda: cache.attend(q.cpu(), table, dl, out), lambda: cache.attend(q.t().contiguous().t(), table, dl, out)):
        with pytest.raises(ValueError):
            f()
    wide = torch.zeros(2, 256 + 12, dtype=torch.bfloat16, device="cuda")
    for f, code in ((lambda: cache.attend(q, table, dl, out, accumulate=True), -1),
                    (lambda: cache.attend(q, table, dl, out, scale=float("nan")), -1),
                    (lambda: cache.attend(wide[:, 4:260], table, dl, out), -1),        # 8-byte aligned
                    (lambda: cache.attend(q, table, dl, wide[:, :256]), -1)):          # stride no multiple of 8
        with pytest.raises(bd.BDLoRAError) as e:
            f()
        assert e.value.code == code
    three = torch.zeros(3, 256, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(bd.BDLoRAError):                                                # more than max_seqs
        cache.attend(three, torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                     torch.zeros_like(three))
    cache.attend(q[:0], table[:0], dl[:0], out[:0])                                    # no sequence: nothing to do
    assert not out.any()
    for kw in ({"page_size": 24}, {"page_size": 8}, {"head_dim": 96}, {"n_q_heads": 3, "n_kv_heads": 2}, {"max_seqs": 0},
               {"fmt": 7}, {"n_pages": 0}):
        a = {"n_q_heads": 4, "n_kv_heads": 2, "head_dim": 64, "n_pages": 4, "page_size": 16, "max_seqs": 2} | kw
        with pytest.raises(bd.BDLoRAError):
            bd.KVCache(**a)
    for kw in ({"k_scale": 0.0}, {"v_scale": float("inf")}, {"k_scale": 0.5}):
        with pytest.raises(bd.BDLoRAError):
            bd.KVCache(4, 2, 64, 4, 16, 2, **kw)
    with pytest.raises(ValueError):
        bd.KVCache(4, 2, 64, 4, 16, 2, k=torch.zeros(4, 2, 16, 64, device="cuda"))
    cache.close()
    with pytest.raises(bd.BDLoRAError):
        cache.attend(q, table, dl, out)


def test_large_values_of_entries_without_probability_add_nothing(torch):
    """An entry whose score is -infinity, or far below the others', has
    probability 0, and 0 times its value is 0, up to the largest number."""
    dc = DrawnCache([40, 40, 3], 1, 64, 16, seed=2)
    for b, n in enumerate(dc.lens):
        k, v = np.zeros((1, n, 64), np.uint16), np.full((1, n, 64), 0x3A80, np.uint16)      # values of 2^-10
        for e, key in ((1, 0xFF80), (2, 0xC700)):            # -infinity, -32768
            k[0, e, 0], v[0, e, :] = key, 0x7F7F             # 3.4e38
            v[0, e, ::2] |= 0x8000
        dc.put(dc.K, b, k)
        dc.put(dc.V, b, v)
    cache, table, dl = dc.device(n_q_heads=4, weights=False)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1.0
    out, lse = torch.empty(3, 256, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 4, device="cuda")
    cache.attend(q.flatten(1), table, dl, out, lse=lse, scale=1.0)
    y = device_to_float(out)
    assert (y == 2.0 ** -10).all(), np.unique(y)
    assert np.allclose(lse.cpu().numpy(), np.log(np.array([38, 38, 1]))[:, None], atol=1e-6)
    cache.close()


@pytest.mark.parametrize("d,fp8", [(64, False), (128, False), (64, True)])
def test_probabilities_keep_the_bits_of_32_in_the_sum_over_values(torch, d, fp8):
    """Sums over values that all but cancel: one entry of probability p (before
    the division) and value 1 (times 256 in 8 bits) beside entries of
    probability 1 whose values are minus the first and the next bits of p (8
    in bf16, 4 in e4m3), so that what is left is p's bits below about 2^-16.

    Tolerance: the score is one product, exact in fp32; its scaling and the
    subtraction round numbers of at most 2 in units of log 2 (2^-24 each of
    it: 2^-23 in all), the exponential to 2^-23, and the sum has at most 9
    terms that are not 0, 2^-23 each: less than 2^-19 of sum p |v|, and the
    store's 2^-8 of the result."""
    B, hq, n = 64, 16, 5
    rng = np.random.default_rng(d + fp8)
    dc = DrawnCache([n] * B, 1, d, 16, seed=1, fp8=fp8)
    qbits, q = wl.bf16_round(rng.uniform(2.0, 9.0, (B, hq)))
    kbits = okv.e4m3_encode(-1.0) if fp8 else 0xBF80
    parts = (lambda x: okv.e4m3_values()[okv.e4m3_encode(x)]) if fp8 else (lambda x: wl.bf16_round(x)[1].astype(np.float64))
    bits = okv.e4m3_encode if fp8 else (lambda x: wl.bf16_round(x)[0])
    full = np.zeros((B, hq, d))
    full[:, :, 0] = q
    for b in range(B):
        K = np.zeros((1, n, d), dc.K.dtype)
        K[0, 1, 0] = kbits
        p = np.exp(-0.125 * q[b].astype(np.float64))
        v = np.zeros((1, n, d))
        v[0, 1, :hq] = 256.0 if fp8 else 1.0
        rest = p * v[0, 1, 0]
        for e in (0, 2, 3, 4) if fp8 else (0, 2):           # columns 0 .. hq - 1, one for each query head
            v[0, e, :hq] = -parts(rest)
            rest = rest + v[0, e, :hq]
        dc.k[b] = okv.e4m3_values()[K].astype(np.float64) if fp8 else wl.bf16_bits_to_float(K).astype(np.float64)
        dc.v[b] = v
        dc.put(dc.K, b, K)
        dc.put(dc.V, b, bits(v).astype(dc.V.dtype))
    cache, table, dl = dc.device(n_q_heads=hq, weights=False)
    qd = torch.from_numpy(wl.bf16_round(full.reshape(B, hq * d))[0].view(np.int16)).cuda().view(torch.bfloat16)
    out = torch.empty(B, hq * d, dtype=torch.bfloat16, device="cuda")
    cache.attend(qd, table, dl, out, scale=0.125)
    y = device_to_float(out).astype(np.float64).reshape(B, hq, d)
    for b in range(B):
        for h in range(hq):
            p = np.exp(0.125 * (dc.k[b][0] @ full[b, h]))
            p /= p.sum()
            ref, mag = p @ dc.v[b][0], p @ np.abs(dc.v[b][0])
            tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * mag
            err = np.abs(y[b, h] - ref)
            assert (err <= tol).all(), (b, h, "times the tolerance: %.2f" % (err[tol > 0] / tol[tol > 0]).max())
    cache.close()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(16, 1, 128), (12, 1, 128), (40, 2, 128), (40, 2, 64), (17, 1, 64)])
def test_many_query_heads_over_long_sequences(torch, hq, hkv, d, fp8):
    """More than 8 query heads a kv head: a workgroup adds its shares in two
    passes, and in groups where a sequence has more than 32 workgroups; more
    than 16: further stretches of the line."""
    lens = [9001, 40001, 8013, 300]
    dc = DrawnCache(lens, hkv, d, 16, seed=hq + d, fp8=fp8, k_scale=0.02 if fp8 else 1.0, v_scale=0.011 if fp8 else 1.0)
    cache, table, dl = dc.device(n_q_heads=hq)
    q, qv = _queries(torch, len(lens), hq, d, seed=hq)
    runs = []
    for i in range(4):
        out = torch.full((len(lens), hq * d), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((len(lens), hq), float("nan"), device="cuda")
        cache.attend(q, table, dl, out, lse=lse, accumulate=i == 0)
        runs.append((out, lse))
    _check(dc, qv, *runs[0], cache.weight, None, d ** -0.5)
    for out, lse in runs[1:]:
        assert torch.equal(out.view(torch.int16), runs[0][0].view(torch.int16)) and torch.equal(lse, runs[0][1])
    assert cache.device_error() == 0
    cache.close()


def test_out_apart_from_the_queries(torch):
    dc = DrawnCache([20, 30], 1, 64, 16, seed=17)
    cache, table, dl = dc.device(n_q_heads=4, weights=False)
    q, _ = _queries(torch, 2, 4, 64, seed=1)
    same = q.clone()
    with pytest.raises(ValueError):
        cache.attend(q, table, dl, q)
    assert torch.equal(q.view(torch.int16), same.view(torch.int16))
    rows = torch.zeros(2, 512, dtype=torch.bfloat16, device="cuda")
    rows[:, :256] = q
    cache.attend(rows[:, :256], table, dl, rows[:, 256:])              # columns of the same rows
    out = torch.empty_like(q)
    cache.attend(q, table, dl, out)
    assert torch.equal(rows[:, 256:].contiguous().view(torch.int16), out.view(torch.int16))
    cache.close()
