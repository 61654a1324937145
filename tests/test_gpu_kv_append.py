"""Rotary embedding and entry of new tokens into the key-value cache.

The rotation is two products and a sum in fp32, each rounded by itself: the
stored numbers are compared bit for bit with the same steps in numpy, and with
the float64 oracle to within their rounding (half a step: bf16, 8 significant
bits, at most 2^-8 of the result; e4m3, 4 bits, 2^-4, or half its smallest
step; and 2^-22 of the products)."""
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


def _tables(d, n):
    a = np.arange(n)[:, None] * (10000.0 ** (-np.arange(d // 2) / (d // 2)))[None, :]
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _f32_rotate(x, c, s, interleaved):
    x = x.astype(np.float32)
    h = x.shape[-1] // 2
    i, j = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, h), slice(h, None))
    y = np.empty_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def _run(torch, dc, hq, seqs, index, positions, interleaved, seed, n_positions=300, weights=True, in_place=False, T_pad=0):
    rng = np.random.default_rng([seed, 1])
    T, d, hkv = len(seqs), dc.d, dc.hkv
    bits, x = wl.bf16_round(rng.standard_normal((T, (hq + 2 * hkv) * d)))
    c, s = _tables(d, n_positions)
    cache, table, lens = dc.device(n_q_heads=hq, weights=weights)
    qkv = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    q_out = qkv[:, :hq * d] if in_place else torch.full((T, hq * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    i32 = lambda v: torch.tensor(np.asarray(v, np.int32), device="cuda")  # noqa: E731
    cache.append(qkv, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), i32(seqs), i32(index), i32(positions), table,
                 lens, q_out, interleaved=interleaved)
    torch.cuda.synchronize()
    return cache, lens, q_out, x.reshape(T, hq + 2 * hkv, d), c, s, qkv, bits


def _check(dc, cache, lens, q_out, x, c, s, hq, seqs, index, positions, interleaved, stored):
    T, hkv, d = len(seqs), dc.hkv, dc.d
    K, V = host_bits(cache.k), host_bits(cache.v)
    wantK, wantV, W, P = dc.K.copy(), dc.V.copy(), dc.W.copy(), dc.P.copy()
    want_lens = dc.lens.copy()
    values = okv.e4m3_values()
    q = device_to_float(q_out).reshape(T, hq, d)
    for t in range(T):
        p = positions[t]
        y = _f32_rotate(x[t, :hq + hkv], c[p], s[p], interleaved)
        assert np.array_equal(q[t], wl.bf16_round(y[:hq])[1]), t
        ref = okv.rotate(x[t, :hq + hkv], c[p].astype(np.float64), s[p].astype(np.float64), interleaved)
        slack = 2.0 ** -22 * 2 * np.abs(x[t, :hq + hkv]).max()
        assert (np.abs(q[t] - ref[:hq]) <= 2.0 ** -8 * np.abs(ref[:hq]) * 1.01 + slack).all(), t
        if not stored[t]:
            continue
        pg, sl = dc.table[seqs[t], index[t] // dc.ps], index[t] % dc.ps
        for want, got, rows, r64, scale in ((wantK, K, y[hq:], ref[hq:], dc.scales[0]),
                                            (wantV, V, x[t, hq + hkv:], x[t, hq + hkv:], dc.scales[1])):
            if dc.fp8:
                inv = np.float32(1) / np.float32(scale)
                want[pg, :, sl] = okv.e4m3_encode((rows.astype(np.float32) * inv).astype(np.float64))
                z = r64 / scale
                e = np.abs(values[got[pg, :, sl]] - np.clip(z, -448, 448))
                assert (e <= 2.0 ** -4 * np.abs(z) * 1.0001 + 2.0 ** -10 + slack / scale).all(), t
            else:
                want[pg, :, sl] = wl.bf16_round(rows)[0]
        W[pg, :, sl] = 0.0
        P[pg, :, sl] = p
        want_lens[seqs[t]] = max(want_lens[seqs[t]], index[t] + 1)
    assert np.array_equal(K, wantK) and np.array_equal(V, wantV)
    assert np.array_equal(lens.cpu().numpy(), want_lens)
    if cache.weight is not None:
        assert np.array_equal(cache.weight.cpu().numpy(), W, equal_nan=True)
        assert np.array_equal(cache.pos.cpu().numpy(), P)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 2), (5, 5)])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_prompts_and_single_tokens(torch, d, hq, hkv, fp8, interleaved):
    # sequence 0: a prompt of 37; 1: a chunk of 20 behind 30 entries; 2-4: one token each; 5: only padding
    lens = [0, 30, 15, 16, 100, 3]
    dc = DrawnCache(lens, hkv, d, 16, seed=d + hq, fp8=fp8, k_scale=0.01 if fp8 else 1.0, v_scale=0.3 if fp8 else 1.0,
                    room=[37, 20, 1, 1, 1, 0])
    seqs = [0] * 37 + [1] * 20 + [2, -1, 3, 4, -1]
    index = list(range(37)) + list(range(30, 50)) + [15, 0, 16, 100, 99999]
    positions = list(range(37)) + list(range(230, 250)) + [15, 0, 299, 7, 31]
    r = _run(torch, dc, hq, seqs, index, positions, interleaved, seed=2)
    _check(dc, *r[:6], hq, seqs, index, positions, interleaved, [q >= 0 for q in seqs])
    assert r[0].device_error() == 0
    r[0].close()


@pytest.mark.parametrize("T", [1, 2, 3, 64, 65, 300])
def test_batch_sizes_pages_and_a_cache_without_weights(torch, T):
    dc = DrawnCache([7 + t % 5 for t in range(T)], 1, 128, 64, seed=T, room=1)
    seqs, index = list(range(T)), [7 + t % 5 for t in range(T)]
    r = _run(torch, dc, 4, seqs, index, index, False, seed=T, weights=False)
    _check(dc, *r[:6], 4, seqs, index, index, False, [True] * T)
    r[0].close()


@pytest.mark.parametrize("interleaved", [False, True])
def test_queries_rotated_in_place(torch, interleaved):
    dc = DrawnCache([4] * 9, 2, 128, 16, seed=5, room=1)
    seqs, index = list(range(9)), [4] * 9
    r = _run(torch, dc, 8, seqs, index, index, interleaved, seed=5, in_place=True)
    _check(dc, r[0], r[1], r[2].contiguous(), *r[3:6], 8, seqs, index, index, interleaved, [True] * 9)
    rest = host_bits(r[6])[:, 8 * 128:]
    assert np.array_equal(rest, r[7][:, 8 * 128:])                 # keys and values stay as they were
    r[0].close()


def test_e4m3_ties_overflow_and_nan(torch):
    dc = DrawnCache([0], 1, 64, 16, seed=6, fp8=True, room=16)
    import paper_2510_23346_amd as bd  # noqa: F401
    v = np.zeros((4, 64), np.float32)
    v[0] = [448, 449, 464, 465, 480, 1e9, -1e9, np.inf, -np.inf, np.nan, 0.0, -0.0] + [0] * 52
    v[1] = np.arange(64) / 64 * 2 + 1              # halfway cases among them
    v[2] = 2.0 ** -9 * (np.arange(64) / 4)         # the smallest steps
    v[3] = -v[1] * 100
    bits = (v.view(np.uint32) >> 16).astype(np.uint16)
    exactv = (bits.astype(np.uint32) << 16).view(np.float32)
    cache, table, lens = dc.device(n_q_heads=1)
    qkv = torch.zeros(4, 192, dtype=torch.bfloat16, device="cuda")
    qkv[:, 128:] = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    c, s = (torch.from_numpy(x).cuda() for x in _tables(64, 8))
    i = torch.arange(4, dtype=torch.int32, device="cuda")
    cache.append(qkv, c, s, torch.zeros_like(i), i, i, table, lens, torch.empty(4, 64, dtype=torch.bfloat16, device="cuda"))
    got = dc.take(host_bits(cache.v), 0, 4)[0]
    want = okv.e4m3_encode(exactv.astype(np.float64))
    nan = np.isnan(exactv)
    assert np.array_equal(got[~nan], want[~nan]) and ((got[nan] & 0x7F) == 0x7F).all()
    cache.close()


def test_what_does_not_fit_is_not_stored_and_raises_the_flag(torch):
    dc = DrawnCache([10, 10, 10], 1, 64, 16, seed=7, room=6, wide=0)
    bad = [(3, 10, 5), (-2, 10, 5), (0, 16, 5), (0, -1, 5), (1, 10, 300), (1, 10, -1), (2, 11, 5)]
    for seq, idx, pos in bad:
        table_hurt = (seq, idx) == (2, 11)
        hurt = DrawnCache([10, 10, 10], 1, 64, 16, seed=7, room=6, wide=0)
        if table_hurt:
            hurt.table[2, 0] = hurt.n_pages
        r = _run(torch, hurt, 2, [seq, 0], [idx, 10], [pos, 10], False, seed=8)
        pos_ok = 0 <= pos < 300
        if not pos_ok:
            q = device_to_float(r[2])
            assert (q[0] == 0).all()
            r[2][0] = torch.from_numpy(wl.bf16_round(_f32_rotate(r[3][0, :2], *(x[0] for x in _tables(64, 300)), False).reshape(-1))[0]
                                       .view(np.int16)).cuda().view(torch.bfloat16)
        _check(hurt, *r[:6], 2, [seq, 0], [idx, 10], [pos if pos_ok else 0, 10], False, [False, True])
        assert r[0].device_error() == 1
        r[0].close()


def test_graph_replay_with_moved_tokens(torch):
    dc = DrawnCache([5, 9, 0], 2, 128, 16, seed=9, room=20)
    rng = np.random.default_rng(1)
    cache, table, lens = dc.device(n_q_heads=4)
    c, s = (torch.from_numpy(x).cuda() for x in _tables(128, 64))
    qkv = torch.from_numpy(rng.standard_normal((3, 8 * 128)).astype(np.float32)).cuda().bfloat16()
    q_out = torch.empty(3, 512, dtype=torch.bfloat16, device="cuda")
    seqs, index = torch.arange(3, dtype=torch.int32, device="cuda"), lens.clone()
    args = (qkv, c, s, seqs, index, index, table, lens, q_out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        cache.append(*args)
    state = [cache.k, cache.v, cache.weight, cache.pos, lens, q_out]
    for rep in range(4):
        before = [x.clone() for x in state]
        g.replay()
        torch.cuda.synchronize()
        after = [x.clone() for x in state]
        for x, y in zip(state, before):
            x.copy_(y)
        cache.append(*args)
        torch.cuda.synchronize()
        for x, y in zip(state, after):
            assert np.array_equal(x.contiguous().view(torch.uint8).cpu().numpy(), y.contiguous().view(torch.uint8).cpu().numpy()), rep
        index += 1
        qkv.mul_(0.5)
    assert lens.tolist() == [9, 13, 4]
    cache.close()


def test_entries_beyond_four_gigabytes(torch):
    import paper_2510_23346_amd as bd
    n_pages, page, d = 90_000, 256, 128
    k = torch.zeros(n_pages, 1, page, d, dtype=torch.bfloat16, device="cuda")        # 5.9 GB each
    v = torch.zeros_like(k)
    cache = bd.KVCache(2, 1, d, n_pages, page, 2, k=k, v=v)
    rng = np.random.default_rng(4)
    bits, x = wl.bf16_round(rng.standard_normal((2, 4 * d)))
    qkv = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    c, s = _tables(d, 8)
    table = torch.tensor([[0, n_pages - 1], [70_001, 3]], dtype=torch.int32, device="cuda")
    i32 = lambda z: torch.tensor(z, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = i32([256, 200])
    cache.append(qkv, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), i32([0, 1]), i32([257, 255]), i32([3, 5]), table,
                 lens, torch.empty(2, 2 * d, dtype=torch.bfloat16, device="cuda"))
    x = x.reshape(2, 4, d)
    for t, (pg, at, p) in enumerate(((n_pages - 1, 1, 3), (70_001, 255, 5))):
        y = _f32_rotate(x[t, 2:3], c[p], s[p], False)
        assert np.array_equal(host_bits(k[pg, 0, at]), wl.bf16_round(y)[0][0])
        assert np.array_equal(host_bits(v[pg, 0, at]), bits.reshape(2, 4, d)[t, 3])
    assert int(torch.count_nonzero(k.view(torch.int16)).item()) <= 2 * d and lens.tolist() == [258, 256]
    cache.close()


def test_refusals(torch):
    import paper_2510_23346_amd as bd
    dc = DrawnCache([4, 4], 1, 64, 16, seed=3, room=1)
    cache, table, lens = dc.device(n_q_heads=2)
    qkv = torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")
    q_out = torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    c, s = (torch.from_numpy(x).cuda() for x in _tables(64, 8))
    i = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ok = dict(qkv=qkv, cos=c, sin=s, seqs=i, index=i, positions=i, table=table, lens=lens, q_out=q_out)
    before = host_bits(cache.k)
    for kw in ({"qkv": qkv.float()}, {"qkv": qkv[:, :255]}, {"cos": c[:, :31]}, {"sin": s[:4]}, {"cos": c.double()},
               {"seqs": i[:1]}, {"index": i.long()}, {"positions": i.cpu()}, {"table": table.float()}, {"lens": lens[:1]},
               {"q_out": q_out[:1]}, {"q_out": q_out.half()}):
        with pytest.raises(ValueError):
            cache.append(**(ok | kw))
    with pytest.raises(bd.BDLoRAError) as e:
        cache.append(**(ok | {"qkv": torch.zeros(2, 260, dtype=torch.bfloat16, device="cuda")[:, 4:]}))
    assert e.value.code == -1
    cache.append(**(ok | {"qkv": qkv[:0], "q_out": q_out[:0], "seqs": i[:0], "index": i[:0], "positions": i[:0]}))
    torch.cuda.synchronize()
    assert np.array_equal(before, host_bits(cache.k)) and cache.device_error() == 0
    cache.append(**(ok | {"lens": None}))
    assert lens.tolist() == [4, 4]
    cache.close()


def test_lens_apart_from_the_integers_that_are_read_beside_it(torch):
    """index and positions of a decode step are the lengths: copies of them."""
    dc = DrawnCache([4, 4], 1, 64, 16, seed=3, room=1)
    cache, table, lens = dc.device(n_q_heads=2)
    qkv, q_out = (torch.zeros(2, n, dtype=torch.bfloat16, device="cuda") for n in (256, 128))
    c, s = (torch.from_numpy(x).cuda() for x in _tables(64, 8))
    both = torch.zeros(4, dtype=torch.int32, device="cuda")
    both[:2] = lens
    lens, after, across = both[:2], both[2:], both[1:3]
    i = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ok = dict(qkv=qkv, cos=c, sin=s, seqs=i, index=lens.clone(), positions=lens.clone(), table=table, lens=lens, q_out=q_out)
    for name in ("seqs", "index", "positions"):
        for x in (lens, across):
            with pytest.raises(ValueError):
                cache.append(**(ok | {name: x}))
    assert lens.tolist() == [4, 4]
    cache.append(**(ok | {"positions": after}))
    assert lens.tolist() == [5, 5] and cache.device_error() == 0
    cache.append(**(ok | {"index": lens, "positions": lens, "lens": None}))         # not written: may be the same
    assert lens.tolist() == [5, 5]
    cache.close()
