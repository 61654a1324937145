"""Attention of many new tokens of each sequence over the paged key-value
cache, and of single tokens beside a window's sinks, against the float64 oracle.

Tolerances (per element, from the formula):
- a score is a sum of d products in fp32: off by at most es = (d + 4) 2^-24
  scale sum |q||k| (and a rounding of the result, and of its exponent);
- a probability is then off by a factor of at most 2 es + 2^-20, its sum of n
  numbers by n 2^-24, and attend_prompt rounds it to bf16 for the sum over
  values: half a step, 2^-8 (attend holds 24 bits);
- out adds one rounding to bf16, 2^-8 of the result.
"""
import numpy as np
import pytest

import workloads as wl
from oracle import kv as okv
from workloads.gpu import device_to_float
from workloads.kv import DrawnCache

pytestmark = pytest.mark.gpu

FORMATS = {"bf16": {}, "fp8": {"fp8": True, "k_scale": 0.015, "v_scale": 0.3}, "int8": {"int8": True}}


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _queries(torch, T, hq, d, seed, scale=2.0):
    bits, x = wl.bf16_round(np.random.default_rng([seed, 5]).standard_normal((T, hq * d)) * scale)
    return torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16), x.astype(np.float64).reshape(T, hq, d)


def _i32(torch, v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _compare(out, lse, q, k, v, scale, seen, bits, what):
    """One sequence's rows: float results against the oracle."""
    hq, d = q.shape[1], q.shape[2]
    ref, rlse, mag = okv.attend_rows(q, k, v, scale, seen)
    G, n = hq // k.shape[0], k.shape[1]
    es = np.zeros((q.shape[0], hq))
    for h in range(hq):
        size = np.abs(q[:, h]) @ np.abs(k[h // G]).T
        es[:, h] = (d + 4) * 2.0 ** -24 * abs(scale) * np.where(seen, size, 0).max(1, initial=0)
    factor = 2.0 ** -bits + 4 * es[..., None] + 2.0 ** -19 + n * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(ref) + factor * mag
    bad = ~(np.abs(out - ref) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], out[bad][:4], ref[bad][:4], tol[bad][:4])
    none = ~seen.any(1)
    assert (out[none] == 0).all() and (lse[none] == -np.inf).all(), what
    d_lse = np.abs(lse[~none] - rlse[~none])
    assert (d_lse <= (2 * es + 2.0 ** -19 + n * 2.0 ** -24 + 2.0 ** -23 * np.abs(np.where(np.isinf(rlse), 0, rlse)))[~none]).all(), what


def _prompt(torch, dc, new, hq, window=0, sinks=0, scale=None, seed=1, behind=0, device=None):
    """A call over the last new[b] entries of the sequences; checks all rows."""
    d, T = dc.d, int(np.sum(new)) + behind
    cache, table, lens = device or dc.device(n_q_heads=hq, weights=False)
    q, x = _queries(torch, T, hq, d, seed)
    out = torch.full((T, hq * d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, hq), 7.0, device="cuda")
    begin = np.concatenate([[0], np.cumsum(new)])
    cache.attend_prompt(q, _i32(torch, begin), table, lens, out, window=window, sinks=sinks, scale=scale, lse=lse)
    assert cache.device_error() == 0
    o, z = device_to_float(out).astype(np.float64).reshape(T, hq, d), lse.cpu().numpy()
    for b, n in enumerate(new):
        if n:
            r = slice(begin[b], begin[b + 1])
            _compare(o[r], z[r], x[r], dc.k[b], dc.v[b], d ** -0.5 if scale is None else scale,
                     okv.sees(int(dc.lens[b]), n, window, sinks), 8, (b, n))
    assert (o[begin[-1]:] == 7.0).all() and (z[begin[-1]:] == 7.0).all()       # rows of no sequence
    return cache, o, z


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (6, 2), (3, 3)])
@pytest.mark.parametrize("page", [16, 64])
def test_lengths_formats_heads(torch, fmt, d, hq, hkv, page):
    #  a whole prompt, one entry, one of many, a chunk, nothing, a few, ends of tiles
    new = [70, 1, 1, 33, 0, 5, 64, 129]
    lens = [70, 1, 130, 100, 50, 16, 64, 200]
    dc = DrawnCache(lens, hkv, d, page, seed=d + hq, **FORMATS[fmt])
    _prompt(torch, dc, new, hq, behind=3)[0].close()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 4), (40, 100), (64, 16), (100, 33), (100, 70), (1000, 9), (0, 50),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
def test_window_and_sinks(torch, fmt, window, sinks):
    new = [300, 1, 37, 130, 2, 0]
    lens = [300, 1, 250, 401, 90, 20]
    dc = DrawnCache(lens, 2, 128, 32, seed=window % 1000, **FORMATS[fmt])
    _prompt(torch, dc, new, 4, window, sinks)[0].close()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (16, 1), (17, 1), (40, 2), (200, 1)])
def test_group_sizes(torch, hq, hkv):
    dc = DrawnCache([50, 9, 100], hkv, 64, 16, seed=hq)
    _prompt(torch, dc, [50, 3, 7], hq, seed=hq)[0].close()
    _prompt(torch, dc, [20, 9, 1], hq, window=11, sinks=3, seed=hq)[0].close()


@pytest.mark.parametrize("B", [1, 63, 64, 65, 200, 256, 257, 700, 2048, 2100])
def test_many_sequences(torch, B):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 90, B)
    new = np.minimum(lens, rng.integers(0, 12, B))
    new[-1:] = lens[-1:]
    dc = DrawnCache(lens, 1, 64, 16, seed=B)
    _prompt(torch, dc, [int(x) for x in new], 4)[0].close()


@pytest.mark.parametrize("d", [64, 128])
def test_long_ones_among_many_sequences(torch, d):
    # (those of 2500 entries are cut into stretches)
    lens = np.random.default_rng(d).integers(1, 60, 300)
    new = np.minimum(lens, np.random.default_rng([d, 1]).integers(0, 30, 300))
    for b, n in ((3, 4), (150, 40), (299, 1)):
        lens[b], new[b] = 2500 + b, n
    dc = DrawnCache(lens, 2, d, 16, seed=d)
    _prompt(torch, dc, [int(x) for x in new], 6, behind=2)[0].close()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("new,length", [(3, 3000), (1, 5000), (130, 2500)])
def test_few_tokens_behind_many_entries(torch, fmt, new, length):
    dc = DrawnCache([length, length - 77, 40], 1, 128, 64, seed=length, **FORMATS[fmt])
    _prompt(torch, dc, [new, min(new, 5), 1], 4)[0].close()
    _prompt(torch, dc, [new, 2, 40], 8, window=1500, sinks=20)[0].close()


def test_a_long_prompt(torch):
    dc = DrawnCache([2100], 2, 128, 64, seed=3)
    _prompt(torch, dc, [2100], 4)[0].close()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1300, 70)])
def test_prompts_whose_last_rows_are_cut_into_stretches(torch, fmt, d, window, sinks):
    dc = DrawnCache([1700, 1300, 90], 1, d, 64, seed=d + window, **FORMATS[fmt])
    _prompt(torch, dc, [1700, 300, 2], 4, window, sinks)[0].close()


def test_pages_beyond_four_gigabytes(torch):
    import paper_2510_23346_amd as bd
    n_pages, page, d = 90_000, 256, 128
    k = torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device="cuda")        # 5.9 GB each
    v = torch.zeros_like(k)
    dc = DrawnCache([700, 300], 1, d, page, seed=15, spare=0)
    at = np.array([n_pages - 1, 0, n_pages - 3, 89_000, 66_000], np.int32)[:dc.n_pages]
    for x, y in ((k, dc.K), (v, dc.V)):
        x[torch.from_numpy(at).cuda().long()] = torch.from_numpy(y.view(np.int16)).cuda().view(torch.bfloat16)
    named = (dc.table >= 0) & (dc.table < dc.n_pages)
    table = _i32(torch, np.where(named, at[np.clip(dc.table, 0, dc.n_pages - 1)], -1))
    cache = bd.KVCache(4, 1, d, n_pages, page, 2, k=k, v=v)
    for new in ([300, 7], [700, 300]):
        _prompt(torch, dc, new, 4, device=(cache, table, _i32(torch, dc.lens)))
    cache.close()


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
def test_scales(torch, scale):
    dc = DrawnCache([150, 30], 1, 64, 16, seed=5)
    _prompt(torch, dc, [100, 30], 2, scale=scale)[0].close()


def test_strides_a_wider_table_and_the_same_bits_again(torch):
    dc = DrawnCache([90, 300], 1, 128, 16, seed=8)
    cache, o, z = _prompt(torch, dc, [90, 200], 4, window=64, sinks=5)
    q, _ = _queries(torch, 290, 4, 128, 1)
    wide = torch.zeros((290, 6 * 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 128:5 * 128] = q
    out = torch.full((290, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    _, table, lens = dc.device(n_q_heads=4, weights=False)
    big = torch.full((2, table.shape[1] + 50), -1, dtype=torch.int32, device="cuda")
    big[:, 50:] = table
    cache.attend_prompt(wide[:, 128:5 * 128], _i32(torch, [0, 90, 290]), big[:, 50:], lens, out[:, 2:6], window=64, sinks=5)
    got = device_to_float(out)
    assert np.array_equal(got[:, 2:6].astype(np.float64), o) and (got[:, :2] == 3).all() and (got[:, 6:] == 3).all()
    cache.close()


def test_what_is_not_seen_may_be_anything(torch):
    # every place outside the windows holds NaN already (DrawnCache); entries
    # before the first token's window, and pages that only they lie in, too
    dc = DrawnCache([400, 260], 1, 128, 16, seed=9)
    for b, (n, new) in enumerate([(400, 30), (260, 1)]):
        first = n - new - 50 + 1
        for stored, plain in ((dc.K, dc.k), (dc.V, dc.v)):
            page, place = dc.where(b)
            stored[page[7:first], :, place[7:first]] = 0x7FC0
        dc.table[b, 1:first // 16] = np.resize([2 ** 31 - 1, -5], first // 16 - 1)
    _prompt(torch, dc, [30, 1], 4, window=50, sinks=7)[0].close()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,length,window", [(20, 20, 0), (7, 150, 0), (300, 310, 0), (300, 310, 40), (150, 150, 9)])
def test_infinite_and_nan_entries_reach_only_the_rows_that_see_them(torch, fmt, d, new, length, window):
    # an entry in the middle of the new tokens: a NaN among its values, then an infinity, then a NaN key; int8: its whole block
    for kind in ("value nan", "value inf", "key nan") if fmt == "bf16" else ("value nan", "key nan"):
        dc = DrawnCache([length, 40], 1, d, 16, seed=length + d, **FORMATS[fmt])
        at = length - new + 2 * new // 3
        page, place = dc.where(0)
        stored, plain = (dc.K, dc.k) if "key" in kind else (dc.V, dc.v)
        if fmt == "int8":
            dc.S[page[at], 0, place[at] // 16, 0 if "key" in kind else 1] = np.nan
            plain[0][0, at // 16 * 16:at // 16 * 16 + 16] = np.nan
        else:
            stored[page[at], 0, place[at], 5] = {"bf16": 0x7F80 if "inf" in kind else 0x7FC0, "fp8": 0x7F}[fmt]
            plain[0][0, at, 5] = np.inf if "inf" in kind else np.nan
        hq, T = 4, new + 40
        cache, table, lens = dc.device(n_q_heads=hq, weights=False)
        q, x = _queries(torch, T, hq, d, 3)
        out, lse = torch.zeros_like(q), torch.zeros((T, hq), device="cuda")
        cache.attend_prompt(q, _i32(torch, [0, new, T]), table, lens, out, window=window, lse=lse)
        o, z = device_to_float(out).astype(np.float64).reshape(T, hq, d), lse.cpu().numpy()
        _compare(o[new:], z[new:], x[new:], dc.k[1], dc.v[1], d ** -0.5, okv.sees(40, 40, window), 8, "other sequence")
        seen = okv.sees(length, new, window)
        hit = seen[:, at // 16 * 16:at // 16 * 16 + 16].any(1) if fmt == "int8" else seen[:, at]
        assert hit.any() and (fmt == "int8" or not hit.all())
        k0, v0 = (np.nan_to_num(y[0], nan=0.0, posinf=0.0) for y in (dc.k, dc.v))
        _compare(o[:new][~hit], z[:new][~hit], x[:new][~hit], k0, v0, d ** -0.5, seen[~hit], 8, kind)
        mine = o[:new][hit]
        if kind == "key nan":
            assert np.isnan(mine).all()
        elif fmt == "int8":
            assert np.isnan(mine).all()
        else:
            # the number's own column is not finite (where its probability is not nothing), the others are right
            assert not np.isfinite(mine[..., 5]).all()
            ref, _, mag = okv.attend_rows(x[:new][hit], k0, v0, d ** -0.5, seen[hit])
            others = np.arange(d) != 5
            tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -7 * mag
            assert (np.abs(mine - ref) <= tol)[..., others].all(), kind
        cache.close()


def test_scores_far_apart_and_infinite(torch):
    dc = DrawnCache([200], 1, 64, 16, seed=10)
    page, place = dc.where(0)
    dc.k[0] *= 0
    dc.K[page, :, place] = 0
    for j, x in ((3, 300.0), (150, 1000.0), (151, -1000.0)):
        dc.k[0][0, j] = x
        dc.K[page[j], 0, place[j]] = wl.bf16_round(np.full(64, x))[0]
    _prompt(torch, dc, [120], 4, seed=2)[0].close()


def test_invalid_arguments_on_the_device(torch):
    dc = DrawnCache([80, 60, 40], 1, 128, 16, seed=11)
    cache, table, lens = dc.device(n_q_heads=4, weights=False)
    q, x = _queries(torch, 100, 4, 128, 3)

    def call(begin, table=table, lens=lens, **more):
        out = torch.full((100, 512), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((100, 4), 7.0, device="cuda")
        cache.attend_prompt(q, _i32(torch, begin), table, lens, out, lse=lse, **more)
        err = cache.device_error()
        return device_to_float(out).astype(np.float64).reshape(100, 4, 128), lse.cpu().numpy(), err

    def right(o, z, b, r0, r1, k=None, v=None):
        _compare(o[r0:r1], z[r0:r1], x[r0:r1], dc.k[b] if k is None else k, dc.v[b] if v is None else v, 128 ** -0.5,
                 okv.sees(dc.lens[b] if k is None else k.shape[1], r1 - r0), 8, b)

    o, z, err = call([0, 80, 90, 100])
    assert err == 0
    right(o, z, 0, 0, 80), right(o, z, 1, 80, 90), right(o, z, 2, 90, 100)
    # rows beyond q, a descending list: what is left of each is computed
    for begin, rows in (([0, 80, 90, 1000], [(0, 0, 80), (1, 80, 90)]), ([0, 80, 60, 70], [(0, 0, 60)]), ([-5, 10, 20, 30], [(1, 10, 20), (2, 20, 30)])):
        o, z, err = call(begin)
        assert err == 1
        for b, r0, r1 in rows:
            if begin[1] == 80 and begin[2] == 60:
                continue                              # rows 60..70 belong to two sequences
            right(o, z, b, r0, r1)
    # more tokens than entries: the first see nothing
    for more in ({}, {"window": 2 ** 31 - 1, "sinks": 2 ** 31 - 1}, {"window": 2 ** 31 - 1}):
        o, z, err = call([0, 0, 0, 100], **more)
        assert err == 1 and (o[:60] == 0).all() and (z[:60] == -np.inf).all()
        right(o, z, 2, 60, 100)
    # lengths beyond the row and below zero
    o, z, err = call([0, 10, 20, 30], lens=_i32(torch, [-3, 60, 40]))
    assert err == 1 and (o[:10] == 0).all()
    right(o, z, 1, 10, 20), right(o, z, 2, 20, 30)
    # a page that is none: its entries are not there
    bad = table.clone()
    bad[1, 1] = dc.n_pages
    o, z, err = call([0, 0, 10, 10], table=bad)
    assert err == 1
    seen = okv.sees(60, 10)
    seen[:, 16:32] = False
    _compare(o[:10], z[:10], x[:10], dc.k[1], dc.v[1], 128 ** -0.5, seen, 8, "page")
    cache.close()


def test_overlapping_rows_leave_the_next_call_right(torch):
    # rows of many sequences on top of each other, more than q has: whatever that
    # gives, the calls behind it, whose sequences are cut into stretches, are right
    dc = DrawnCache([3000, 1100], 1, 64, 16, seed=13)
    cache, table, lens = dc.device(n_q_heads=4, weights=False, max_seqs=600)
    q, x = _queries(torch, 100, 4, 64, 2)
    out = torch.zeros_like(q)
    tables, lengths = table[:1].repeat(600, 1), lens[:1].repeat(600)
    for rows in (100, 8):
        cache.attend_prompt(q, _i32(torch, [0, rows] * 300 + [0]), tables, lengths, out)
        assert cache.device_error() == 1
        for new in ([100, 70], [3, 5]):
            _prompt(torch, dc, new, 4, device=(cache, table, lens))
    cache.close()


def test_another_stream_and_graph_replays(torch):
    dc = DrawnCache([300, 120, 500], 2, 128, 64, seed=12, int8=True)
    cache, table, lens = dc.device(n_q_heads=8)
    q, x = _queries(torch, 400, 8, 128, 6)
    begin = _i32(torch, [0, 100, 220, 400])
    out, lse = torch.zeros_like(q), torch.zeros((400, 8), device="cuda")
    eager = []
    batches = [([0, 100, 220, 400], [300, 120, 500]), ([0, 1, 2, 300], [299, 3, 299]), ([0, 0, 64, 64], [7, 64, 0])]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for b, n in batches:
        begin.copy_(_i32(torch, b)), lens.copy_(_i32(torch, n)), out.zero_(), lse.zero_()
        torch.cuda.synchronize()
        cache.attend_prompt(q, begin, table, lens, out, window=200, sinks=3, lse=lse, stream=side)
        torch.cuda.synchronize()
        eager.append((out.clone(), lse.clone()))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.attend_prompt(q, begin, table, lens, out, window=200, sinks=3, lse=lse)
    for turn in range(2):
        for (b, n), (o, z) in zip(batches, eager):
            begin.copy_(_i32(torch, b)), lens.copy_(_i32(torch, n)), out.zero_(), lse.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, o) and torch.equal(lse, z)
    assert cache.device_error() == 0
    del g
    cache.close()


def test_refusals(torch):
    import paper_2510_23346_amd as bd
    cache = bd.KVCache(4, 1, 128, 8, 16, 2)
    q = torch.zeros((6, 512), dtype=torch.bfloat16, device="cuda")
    out, table = torch.zeros_like(q), torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    lens, begin = _i32(torch, [6, 6]), _i32(torch, [0, 3, 6])
    ok = dict(q=q, q_starts=begin, table=table, lens=lens, out=out)
    cache.attend_prompt(**ok)
    for change in (dict(q=q.float()), dict(q=q[:, :500]), dict(q=q.cpu()), dict(out=q), dict(out=out[:5]), dict(q_starts=begin[:2]),
                   dict(q_starts=begin.long()), dict(q_starts=begin.cpu()), dict(lens=lens.long()), dict(table=table[:1]),
                   dict(lse=torch.zeros((6, 3), device="cuda")), dict(window=2 ** 31), dict(sinks=2 ** 31),
                   dict(q=torch.zeros((6, 1024), dtype=torch.bfloat16, device="cuda")[:, ::2])):
        with pytest.raises(ValueError):
            cache.attend_prompt(**{**ok, **change})
    for change in (dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(lens=_i32(torch, [1] * 3), q_starts=_i32(torch, [0] * 4)),
                   dict(q=torch.zeros((6, 516), dtype=torch.bfloat16, device="cuda")[:, :512]),
                   dict(q=torch.zeros(6 * 512 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(6, 512))):
        with pytest.raises(bd.BDLoRAError):
            cache.attend_prompt(**{**ok, **change})
    cache.attend_prompt(q[:0], _i32(torch, [0, 0, 0]), table, lens, out[:0])
    cache.attend_prompt(q, _i32(torch, [0]), table, lens[:0], out)
    torch.cuda.synchronize()
    cache.close()


# ------------------------------------------------ single tokens beside sinks

@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sinks", [0, 1, 15, 16, 20, 40, 1000])
def test_single_tokens_with_sinks(torch, fmt, d, sinks):
    lens = [0, 1, 17, 64, 100, 333, 700, 1500, 45]
    starts = [0, 0, 5, 64, 38, 300, 31, 1499, 50]
    hq, hkv = 6, 2
    dc = DrawnCache(lens, hkv, d, 32, seed=sinks, **FORMATS[fmt])
    weights = fmt != "int8"
    cache, table, dl = dc.device(n_q_heads=hq, weights=weights)
    q, x = _queries(torch, len(lens), hq, d, sinks)
    out, lse = torch.empty_like(q), torch.empty((len(lens), hq), device="cuda")
    cache.attend(q, table, dl, out, starts=_i32(torch, starts), lse=lse, sinks=sinks, accumulate=weights)
    assert cache.device_error() == 0
    o, z = device_to_float(out).astype(np.float64).reshape(-1, 1, hq, d), lse.cpu().numpy()
    W = cache.weight.cpu().numpy() if weights else None
    for b, (n, s) in enumerate(zip(lens, starts)):
        j = np.arange(n)
        seen = ((j >= s) | (j < sinks))[None, :]
        _compare(o[b], z[b:b + 1], x[b:b + 1], dc.k[b], dc.v[b], d ** -0.5, seen, 15, b)
        if weights and n:
            p = np.zeros((hkv, n))
            for h in range(hq):
                a = np.where(seen[0], d ** -0.5 * (dc.k[b][h // 3] @ x[b, h]), -np.inf)
                if seen.any():
                    p[h // 3] += np.exp(a - a.max()) / np.exp(a - a.max()).sum()
            want = dc.weight[b] + p
            # a probability is off by 2 es + 2^-19, es as above, and the sum by its roundings
            es = (d + 4) * 2.0 ** -24 * d ** -0.5 * max((np.abs(dc.k[b][h // 3]) @ np.abs(x[b, h])).max() for h in range(hq))
            assert (np.abs(dc.take(W, b, n) - want) <= (4 * es + 2.0 ** -18) * p + 2.0 ** -22 * want).all(), b
    cache.close()


@pytest.mark.parametrize("fmt", list(FORMATS))
def test_long_sequences_with_sinks_join(torch, fmt):
    # many workgroups a sequence, the gap in the middle of them
    lens, starts = [6000, 900, 4100], [2500, 890, 70]
    dc = DrawnCache(lens, 1, 128, 64, seed=4, **FORMATS[fmt])
    cache, table, dl = dc.device(n_q_heads=20, weights=False)
    q, x = _queries(torch, 3, 20, 128, 9)
    for sinks in (0, 64, 900):
        out, lse = torch.empty_like(q), torch.empty((3, 20), device="cuda")
        cache.attend(q, table, dl, out, starts=_i32(torch, starts), lse=lse, sinks=sinks)
        o, z = device_to_float(out).astype(np.float64).reshape(-1, 1, 20, 128), lse.cpu().numpy()
        for b, (n, s) in enumerate(zip(lens, starts)):
            j = np.arange(n)
            _compare(o[b], z[b:b + 1], x[b:b + 1], dc.k[b], dc.v[b], 128 ** -0.5, ((j >= s) | (j < sinks))[None, :], 15, b)
    cache.close()


def test_sinks_without_starts_change_nothing_and_the_gap_may_be_anything(torch):
    dc = DrawnCache([500, 300], 1, 128, 16, seed=13)
    cache, table, dl = dc.device(n_q_heads=4, weights=False)
    q, x = _queries(torch, 2, 4, 128, 10)
    a, b = torch.empty_like(q), torch.empty_like(q)
    cache.attend(q, table, dl, a)
    cache.attend(q, table, dl, b, sinks=5)
    assert torch.equal(a, b)
    cache.close()
    for i, (n, first) in enumerate([(500, 400), (300, 290)]):
        page, place = dc.where(i)
        dc.K[page[5:first], :, place[5:first]] = dc.V[page[5:first], :, place[5:first]] = 0x7FC0
        dc.table[i, 1:first // 16] = -9
    cache, table, dl = dc.device(n_q_heads=4, weights=False)
    out, lse = torch.empty_like(q), torch.empty((2, 4), device="cuda")
    cache.attend(q, table, dl, out, starts=_i32(torch, [400, 290]), lse=lse, sinks=5)
    assert cache.device_error() == 0
    o, z = device_to_float(out).astype(np.float64).reshape(-1, 1, 4, 128), lse.cpu().numpy()
    for i, (n, first) in enumerate([(500, 400), (300, 290)]):
        j = np.arange(n)
        _compare(o[i], z[i:i + 1], x[i:i + 1], dc.k[i], dc.v[i], 128 ** -0.5, ((j >= first) | (j < 5))[None, :], 15, i)
    with pytest.raises(Exception):
        cache.attend(q, table, dl, out, starts=_i32(torch, [400, 290]), sinks=-1)
    cache.close()
