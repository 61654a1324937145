"""Entry of new tokens with norms of their heads, the 8-bit cache with a scale for
each block, and entries read back.

Without norms the stored integers and scales are compared bit for bit with the
same fp32 steps in numpy.  With them (float64 oracle): the mean square of d
numbers in fp32 is off by at most (d + 2) 2^-24 of itself, so its root's inverse
by half of that and 3 roundings, a normed number by (d / 2 + 6) 2^-24 of itself,
a rotated one by e = (d / 2 + 9) 2^-24 of |x1| + |x2|; bf16 adds half a step,
2^-8, e4m3 2^-4 (or half its smallest step), an integer half a scale."""
import numpy as np
import pytest

import workloads as wl
from oracle import kv as okv
from workloads.gpu import device_to_float
from workloads.kv import DrawnCache, host_bits

pytestmark = pytest.mark.gpu

f32 = np.float32


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _i32(torch, v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _tables(d, n):
    a = np.arange(n)[:, None] * (10000.0 ** (-np.arange(d // 2) / (d // 2)))[None, :]
    return np.cos(a).astype(f32), np.sin(a).astype(f32)


def _f32_rotate(x, c, s, interleaved):
    h = x.shape[-1] // 2
    i, j = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, h), slice(h, None))
    y = np.empty_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


class Stored:
    """A device cache, and what its int8 numbers have to be."""

    def __init__(self, torch, dc, hq, n_positions=300):
        self.torch, self.dc, self.hq = torch, dc, hq
        self.cache, self.table, self.lens = dc.device(n_q_heads=hq)
        self.cos, self.sin = _tables(dc.d, n_positions)
        self.dev = [torch.from_numpy(x).cuda() for x in (self.cos, self.sin)]
        self.K, self.V, self.S, self.want_lens = dc.K.copy(), dc.V.copy(), dc.S.copy(), dc.lens.copy()

    def append(self, seqs, index, positions, seed, interleaved=False, change=None, stored=None, size=1.0):
        torch, dc, hq = self.torch, self.dc, self.hq
        T, d, hkv = len(seqs), dc.d, dc.hkv
        x = np.random.default_rng([seed, 1]).standard_normal((T, hq + 2 * hkv, d)) * size
        if change:
            change(x)
        bits, x = wl.bf16_round(x.reshape(T, -1))
        x = x.reshape(T, -1, d).astype(f32)
        qkv = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
        q_out = torch.full((T, hq * d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.cache.append(qkv, *self.dev, _i32(torch, seqs), _i32(torch, index), _i32(torch, positions), self.table, self.lens, q_out,
                          interleaved=interleaved)
        stored = [s >= 0 for s in seqs] if stored is None else stored
        ok = [0 <= p < len(self.cos) for p in positions]
        at = np.where(ok, positions, 0)
        y = _f32_rotate(x[:, :hq + hkv], self.cos[at][:, None], self.sin[at][:, None], interleaved)
        y[~np.array(ok)] = 0
        assert np.array_equal(device_to_float(q_out).reshape(T, hq, d), wl.bf16_round(y[:, :hq])[1])
        for b in sorted(set(s for s, k in zip(seqs, stored) if k)):
            ts = [t for t in range(T) if seqs[t] == b and stored[t]]
            n = (max(index[t] for t in ts) // 16 + 1) * 16
            j = np.arange(n)
            page, place = dc.table[b, j // dc.ps], j % dc.ps
            for h in range(hkv):
                for pages, rows, which in ((self.K, y[:, hq + h], 0), (self.V, x[:, hq + hkv + h], 1)):
                    q, s = pages[page, h, place], self.S[page[::16], h, place[::16] // 16, which]
                    okv.int8_blocks(q, s, rows[ts], [index[t] for t in ts])
                    pages[page, h, place] = q
                    self.S[page[::16], h, place[::16] // 16, which] = s
            self.want_lens[b] = max(self.want_lens[b], max(index[t] for t in ts) + 1)

    def check(self, err=0):
        self.torch.cuda.synchronize()
        assert np.array_equal(self.cache.scales.cpu().numpy(), self.S, equal_nan=True)
        assert np.array_equal(self.cache.k.cpu().numpy(), self.K) and np.array_equal(self.cache.v.cpu().numpy(), self.V)
        assert np.array_equal(self.lens.cpu().numpy(), self.want_lens)
        assert self.cache.device_error() == err


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 2), (5, 5), (40, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_prompts_chunks_and_single_tokens(torch, d, hq, hkv, interleaved):
    # a prompt of 37; a chunk of 20 behind 30 entries; single tokens at the ends and in the middle of blocks; padding
    dc = DrawnCache([0, 30, 15, 16, 100, 3, 47], hkv, d, 16, seed=d + hq, int8=True, room=[37, 20, 1, 1, 1, 0, 2])
    s = Stored(torch, dc, hq)
    s.append([0] * 37 + [1] * 20 + [2, -1, 3, 4, -1, 6, 6], list(range(37)) + list(range(30, 50)) + [15, 0, 16, 100, 99999, 47, 48],
             list(range(37)) + list(range(230, 250)) + [15, 0, 299, 7, 31, 1, 2], 1, interleaved)
    s.check()
    s.cache.close()


@pytest.mark.parametrize("page", [16, 64, 256])
def test_steps_whose_scales_grow(torch, page):
    dc = DrawnCache([0, 5, 16], 2, 128, page, seed=page, int8=True, room=60)
    s = Stored(torch, dc, 4)
    at = [0, 5, 16]
    for step in range(40):
        s.append([0, 1, 2], at, at, step, size=np.array([1.0, 1.0 + step, 20.0 / (1 + step)])[:, None, None])
        at = [i + 1 for i in at]
    s.check()
    # written again in the middle of a block, as after tokens that were taken back
    s.append([1, 1, 0], [34, 35, 3], [34, 35, 3], 99, size=100.0)
    s.check()
    s.cache.close()


@pytest.mark.parametrize("T", [1, 3, 64, 65, 300])
def test_batch_sizes(torch, T):
    dc = DrawnCache([7 + t % 20 for t in range(T)], 1, 128, 64, seed=T, int8=True, room=1)
    s = Stored(torch, dc, 4)
    s.append(list(range(T)), [7 + t % 20 for t in range(T)], [t % 300 for t in range(T)], T)
    s.check()
    s.cache.close()


@pytest.mark.parametrize("d", [64, 128])
def test_long_prompts(torch, d):
    # runs that begin anywhere in a block, single tokens and padding between them, a position outside in the middle of one
    dc = DrawnCache([0, 5, 31, 0, 48], 2, d, 64, seed=d, int8=True, room=[1000, 901, 300, 17, 1])
    s = Stored(torch, dc, 4, n_positions=1001)
    seqs = [0] * 1000 + [-1] * 3 + [1] * 901 + [4] + [2] * 300 + [3] * 17 + [-1]
    index = list(range(1000)) + [0, 1, 2] + list(range(5, 906)) + [48] + list(range(31, 331)) + list(range(17)) + [17]
    positions = list(index)
    positions[1500] = 1001
    stored = [b >= 0 and positions[t] < 1001 for t, b in enumerate(seqs)]
    assert len(seqs) == len(index) == 2223
    s.append(seqs, index, positions, 1, stored=stored)
    s.check(err=1)
    s.cache.close()


def test_many_heads_of_prompts_and_single_tokens(torch):
    lens = [0, 70] + [3 + t % 40 for t in range(230)]
    dc = DrawnCache(lens, 8, 64, 16, seed=6, int8=True, room=[400, 411] + [1] * 230)
    s = Stored(torch, dc, 8, n_positions=500)
    seqs = [0] * 400 + list(range(2, 100)) + [1] * 411 + list(range(100, 232))
    index = list(range(400)) + lens[2:100] + list(range(70, 481)) + lens[100:]
    for step in range(2):
        s.append(seqs, index, index, step, size=1.0 + step)
        s.check()
    s.cache.close()


def test_tokens_that_are_not_stored(torch):
    # positions and places outside, in the middle of a run; a page that is none; zeros
    dc = DrawnCache([0, 10, 20, 40], 1, 64, 16, seed=3, int8=True, room=40)
    dc.table[3, 3] = -1
    s = Stored(torch, dc, 4)

    def zero(x):
        x[20:22] = 0

    s.append([0] * 20 + [1, 1, 2, 2, 9, 3, 3, -1], list(range(20)) + [10, 11, 20, 2 ** 30, 3, 47, 48, 1],
             list(range(7)) + [300, -1] + list(range(9, 20)) + [10, 11, 20, 3, 3, 4, 5, 6], 4, change=zero,
             stored=[t not in (7, 8) for t in range(20)] + [True, True, True, False, False, True, False, False])
    s.check(err=1)
    s.cache.close()


def test_a_block_of_nan(torch):
    dc = DrawnCache([16, 20, 18], 1, 64, 16, seed=4, int8=True, room=20)
    cache, table, lens = dc.device(n_q_heads=2)
    c, s = (torch.from_numpy(x).cuda() for x in _tables(64, 100))
    qkv = torch.ones((3, 4 * 64), dtype=torch.bfloat16, device="cuda")
    qkv[0, 130], qkv[1, 200], qkv[2, 255] = float("nan"), float("inf"), -float("inf")     # key, value, value
    cache.append(qkv, c, s, _i32(torch, [0, 1, 2]), _i32(torch, [16, 20, 18]), _i32(torch, [0, 0, 0]), table, lens, qkv[:, :128])
    k, v = (torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(_i32(torch, [0, 1, 2]), _i32(torch, [16, 16, 17]), table, k, v)
    k, v = device_to_float(k), device_to_float(v)
    assert np.isnan(k[0]).all() and np.isfinite(k[1:]).all() and np.isfinite(v[0]).all() and np.isnan(v[1:]).all()
    # it stays so until the block begins anew
    qkv.fill_(1.0)
    for i, nan in ((17, True), (16, False)):
        cache.append(qkv[:1], c, s, _i32(torch, [0]), _i32(torch, [i]), _i32(torch, [0]), table, lens, qkv[:1, :128])
        out = torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda")
        cache.read(_i32(torch, [0]), _i32(torch, [i]), table, out, torch.zeros_like(out))
        assert bool(torch.isnan(out).all()) == nan
    cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("d,hkv,page", [(64, 1, 16), (128, 2, 64), (128, 33, 16), (64, 3, 256)])
def test_read(torch, fmt, d, hkv, page):
    lens = [5, 100, 0, 33]
    dc = DrawnCache(lens, hkv, d, page, seed=d + hkv, fp8=fmt == "fp8", k_scale=0.3 if fmt == "fp8" else 1.0,
                    v_scale=0.7 if fmt == "fp8" else 1.0, int8=fmt == "int8")
    cache, table, _ = dc.device()
    rng = np.random.default_rng(1)
    seqs = rng.choice([0, 1, 3, -1], 301)
    index = np.array([rng.integers(0, lens[b]) if b >= 0 else 12345678 for b in seqs])
    wide = torch.full((2, 301, hkv * d + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = wide[0, :, 8:8 + hkv * d], wide[1, :, 8:8 + hkv * d]
    cache.read(_i32(torch, seqs), _i32(torch, index), table, k, v)
    for got, plain in ((k, dc.k), (v, dc.v)):
        got = device_to_float(got.contiguous()).reshape(301, hkv, d)
        for t, (b, j) in enumerate(zip(seqs, index)):
            # (a product of 8-bit numbers with an fp32 scale is exact in float64 and, but
            # for one rounding to fp32, in fp32: the two roundings are those of the kernel)
            want = wl.bf16_round(plain[b][:, j].astype(f32))[1] if b >= 0 else np.zeros((hkv, d))
            assert np.array_equal(got[t], want), t
    assert (wide[:, :, :8] == 7).all() and (wide[:, :, 8 + hkv * d:] == 7).all()
    assert cache.device_error() == 0
    # what names no entry
    cache.read(_i32(torch, [4, 1, 1, -2]), _i32(torch, [0, -1, 2 ** 30, 0]), table, k[:4], v[:4])
    assert cache.device_error() == 1 and not k[:4].any() and not v[:4].any()
    cache.read(_i32(torch, []), _i32(torch, []), table, k[:0], v[:0])
    cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (6, 3), (64, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norms(torch, fmt, d, hq, hkv, interleaved):
    eps = 1e-5
    lens = [0, 30, 15, 100]
    dc = DrawnCache(lens, hkv, d, 16, seed=d, fp8=fmt == "fp8", k_scale=0.02 if fmt == "fp8" else 1.0, v_scale=0.3 if fmt == "fp8" else 1.0,
                    int8=fmt == "int8", room=[20, 3, 1, 1])
    cache, table, dl = dc.device(n_q_heads=hq, weights=fmt == "bf16")
    seqs, index = [0] * 20 + [1] * 3 + [-1, 2, 3], list(range(20)) + [30, 31, 32, 0, 15, 100]
    pos = [(7 * t) % 300 for t in range(26)]
    rng = np.random.default_rng([d, 2])
    size = np.exp(3 * rng.standard_normal((26, hq + 2 * hkv, 1)))
    size[3] = 0                                             # a row of zeros, and one that eps decides
    size[4] = 1e-3
    bits, x = wl.bf16_round((rng.standard_normal((26, hq + 2 * hkv, d)) * size).reshape(26, -1))
    wb, w = wl.bf16_round(1 + 0.5 * rng.standard_normal((2, d)))
    dev = lambda b: torch.from_numpy(b.view(np.int16).copy()).cuda().view(torch.bfloat16)  # noqa: E731
    c, s = _tables(d, 300)
    qkv = dev(bits)
    cache.append(qkv, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), _i32(torch, seqs), _i32(torch, index), _i32(torch, pos), table, dl,
                 qkv[:, :hq * d], interleaved=interleaved, q_norm=dev(wb[0]), k_norm=dev(wb[1]), eps=eps)
    x = x.reshape(26, -1, d).astype(np.float64)
    normed = np.concatenate([okv.head_norm(x[:, :hq], w[0], eps), okv.head_norm(x[:, hq:hq + hkv], w[1], eps)], 1)
    ref = okv.rotate(normed, c[pos][:, None].astype(np.float64), s[pos][:, None].astype(np.float64), interleaved)
    h = d // 2
    pair = np.repeat(np.abs(normed[..., 0::2]) + np.abs(normed[..., 1::2]), 2, -1) if interleaved else \
        np.tile(np.abs(normed[..., :h]) + np.abs(normed[..., h:]), 2)
    e = (d / 2 + 9) * 2.0 ** -24 * pair
    got = device_to_float(qkv[:, :hq * d].contiguous()).reshape(26, hq, d)
    assert (np.abs(got - ref[:, :hq]) <= 2.0 ** -8 * np.abs(ref[:, :hq]) * 1.01 + e[:, :hq]).all()
    k = torch.zeros((26, hkv * d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    cache.read(_i32(torch, seqs), _i32(torch, index), table, k, v)
    k, v = (device_to_float(t).reshape(26, hkv, d).astype(np.float64) for t in (k, v))
    S = cache.scales.cpu().numpy().astype(np.float64) if fmt == "int8" else None
    for t in range(26):
        if seqs[t] < 0:
            continue
        for got, want, off, which in ((k[t], ref[t, hq:], e[t, hq:], 0), (v[t], x[t, hq + hkv:], 0, 1)):
            if fmt == "bf16":
                tol = 2.0 ** -8 * np.abs(want) * 1.01 + off
                if which:
                    tol = 0
            elif fmt == "fp8":
                scale = dc.scales[which]
                want = np.clip(want, -448 * scale, 448 * scale)
                tol = (2.0 ** -4 + 2.0 ** -8) * np.abs(want) * 1.01 + 2.0 ** -10 * scale + off
            else:
                f = S[dc.table[seqs[t], index[t] // 16], :, 0, which][:, None]
                tol = 0.5 * f * (1 + 2.0 ** -14) + 2.0 ** -8 * (np.abs(want) + f) + off
            assert (np.abs(got - want) <= tol).all(), (t, which)
    assert np.array_equal(dl.cpu().numpy(), [20, 33, 16, 101]) and cache.device_error() == 0
    cache.close()


def test_norms_leave_the_rest_as_it_was(torch):
    # a norm of weight 1 and mean square 1 - eps: the call without norms, up to roundings of fp32
    dc = DrawnCache([0], 1, 128, 16, seed=1, room=33)
    a, table, la = dc.device(n_q_heads=4, weights=False)
    b, _, lb = dc.device(n_q_heads=4, weights=False)
    c, s = (torch.from_numpy(x).cuda() for x in _tables(128, 40))
    qkv = torch.sign(torch.randn((33, 6 * 128), device="cuda")).to(torch.bfloat16)
    one = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    i = _i32(torch, range(33))
    qa, qb = (torch.empty((33, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a.append(qkv, c, s, i * 0, i, i, table, la, qa)
    b.append(qkv, c, s, i * 0, i, i, table, lb, qb, q_norm=one, k_norm=one, eps=0.0)
    assert torch.equal(qa, qb) and np.array_equal(host_bits(a.k), host_bits(b.k)) and torch.equal(la, lb)
    a.close(), b.close()


def test_refusals(torch):
    import paper_2510_23346_amd as bd
    with pytest.raises(ValueError):
        bd.KVCache(4, 1, 128, 8, 16, 2, fmt=bd.KV_INT8, weights=True)
    with pytest.raises(ValueError):
        bd.KVCache(4, 1, 128, 8, 16, 2, scales=torch.zeros((8, 1, 1, 2), device="cuda"))
    for bad in (torch.zeros((8, 1, 2, 2), device="cuda"), torch.zeros((8, 1, 1, 2)), torch.zeros((8, 1, 1, 2), device="cuda").half()):
        with pytest.raises(ValueError):
            bd.KVCache(4, 1, 128, 8, 16, 2, fmt=bd.KV_INT8, scales=bad)
    with pytest.raises(bd.BDLoRAError):
        bd.KVCache(4, 1, 128, 8, 16, 2, fmt=bd.KV_INT8, k_scale=0.5)
    cache = bd.KVCache(4, 1, 128, 8, 16, 2, fmt=bd.KV_INT8)
    table, lens = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), _i32(torch, [4, 4])
    q = torch.zeros((2, 512), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(bd.BDLoRAError):
        cache.evict(table, lens, 2)
    with pytest.raises(bd.BDLoRAError):
        cache.attend(q, table, lens, torch.empty_like(q), accumulate=True)
    k, v = (torch.zeros((2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i = _i32(torch, [0, 1])
    with pytest.raises(bd.BDLoRAError):
        cache.read(i, i, table, k, k)
    for change in (dict(k_out=k[:1]), dict(v_out=v.float()), dict(seqs=i[:1]), dict(index=i.long()), dict(table=table.cpu())):
        with pytest.raises(ValueError):
            cache.read(**{**dict(seqs=i, index=i, table=table, k_out=k, v_out=v), **change})
    c = torch.zeros((10, 64), device="cuda")
    qkv = torch.zeros((2, 768), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(q_norm=w), dict(k_norm=w), dict(q_norm=w.float(), k_norm=w), dict(q_norm=w[:64], k_norm=w),
                dict(q_norm=w, k_norm=torch.ones(256, dtype=torch.bfloat16, device="cuda")[::2])):
        with pytest.raises(ValueError):
            cache.append(qkv, c, c, i, i, i, table, lens, q, **bad)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(bd.BDLoRAError):
            cache.append(qkv, c, c, i, i, i, table, lens, q, q_norm=w, k_norm=w, eps=eps)
    cache.close()


def test_entries_beyond_four_gigabytes(torch):
    # 640 pages of 65536 entries of 128 bytes: 5.4 GB each of keys and values
    import paper_2510_23346_amd as bd
    n, ps = 640, 65536
    k, v = (torch.empty((n, 1, ps, 128), dtype=torch.int8, device="cuda") for _ in range(2))
    scales = torch.full((n, 1, ps // 16, 2), float("nan"), device="cuda")
    cache = bd.KVCache(4, 1, 128, n, ps, 2, fmt=bd.KV_INT8, k=k, v=v, scales=scales)
    rng = np.random.default_rng(1)
    T = 150
    bits, x = wl.bf16_round(rng.standard_normal((T, 6 * 128)))
    qkv = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    c, s = torch.ones((1, 64), device="cuda"), torch.zeros((1, 64), device="cuda")
    table, lens = _i32(torch, [[639, 5], [638, 600]]), _i32(torch, [0, 0])
    i, z = _i32(torch, range(T)), _i32(torch, [0] * T)
    cache.append(qkv, c, s, z, i, z, table, lens, qkv[:, :512])
    ko, vo = (torch.zeros((T, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(z, i, table, ko, vo)
    x = x.reshape(T, 6, 128).astype(np.float64)
    for got, want in ((ko, x[:, 4]), (vo, x[:, 5])):
        d = np.abs(device_to_float(got) - want)
        top = np.repeat([np.abs(want[b:b + 16]).max() for b in range(0, T, 16)], 16)[:T, None]
        assert (d <= top / 127 * 0.5 * 1.001 + 2.0 ** -8 * (np.abs(want) + top / 127)).all()
    kk, vv = device_to_float(ko).astype(np.float64), device_to_float(vo).astype(np.float64)
    out, one = torch.empty((T, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((1, 512), dtype=torch.bfloat16, device="cuda")
    cache.attend_prompt(qkv[:, :512], _i32(torch, [0, T]), table, lens[:1], out)
    cache.attend(qkv[-1:, :512], table, lens[:1], one)
    ref, _, mag = okv.attend_rows(x[:, :4], kk[None], vv[None], 128 ** -0.5, okv.sees(T, T))
    # (keys and values taken back are rounded to bf16: 2^-8 of each, a score by 2^-8 scale sum |q||k|)
    es = 2.0 ** -8 * 128 ** -0.5 * np.stack([(np.abs(x[:, h]) @ np.abs(kk).T).max(1) for h in range(4)], 1)[..., None]
    tol = 2.0 ** -8 * np.abs(ref) + (2 * es + 2.0 ** -7 + 2.0 ** -12) * 1.05 * mag
    assert (np.abs(device_to_float(out).reshape(T, 4, 128) - ref) <= tol).all()
    assert (np.abs(device_to_float(one).reshape(4, 128) - ref[-1]) <= tol[-1]).all()
    assert cache.device_error() == 0
    cache.close()
