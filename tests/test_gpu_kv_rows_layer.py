"""A layer's attention block with norms, a window and sinks over each cache format:
prompts in chunks, then steps (eager, and as a captured graph replayed beside
eager work), every stage against the float64 oracle on what the stage before it
left; and the cache's calls in other orders and on several streams.

Tolerances: the projections are held to the library's rule (1e-2, as in
test_gpu_kv_layer.py); attention as in test_gpu_kv_prompt.py, on the entries
that read gives back, which are rounded to bf16 once more in an 8-bit cache
(2^-8 of each key and value: a score by 2^-8 scale sum |q||k|, out by 2^-8 sum
p |v|)."""
import os
import sys

import numpy as np
import pytest

import workloads as wl
from oracle import bdlora, kv as okv
from workloads.gpu import device_to_float

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _i32(torch, v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _held(torch, block, b, n):
    """Entries of sequence b as read gives them back: k, v [heads, n, d]."""
    c = block.cache
    k, v = (torch.zeros((n, c.n_kv_heads * c.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.read(_i32(torch, [b] * n), _i32(torch, range(n)), block.table, k, v)
    return [device_to_float(t).astype(np.float64).reshape(n, c.n_kv_heads, c.head_dim).transpose(1, 0, 2) for t in (k, v)]


def _attention(q, k, v, seen, got, what):
    d = q.shape[2]
    ref, _, mag = okv.attend_rows(q, k, v, d ** -0.5, seen)
    G = q.shape[1] // k.shape[0]
    size = np.stack([np.where(seen, np.abs(q[:, h]) @ np.abs(k[h // G]).T, 0).max(1) for h in range(q.shape[1])], 1)
    es = 2.0 ** -8 * d ** -0.5 * size[..., None] * 1.01
    tol = 2.0 ** -8 * np.abs(ref) + (np.expm1(2 * es) + 2.0 ** -7 + 2.0 ** -12) * 1.01 * mag
    assert (np.abs(got - ref) <= tol).all(), what


def _project(block, p, x, slots):
    y = x @ device_to_float(block.w[p]).astype(np.float64).T
    for t, a in enumerate(slots):
        A, B = block.adapters[a]
        at = 0
        for s, n in enumerate((block.qkv, block.o)[p].slices):
            y[t, at:at + n] += 2.0 * (x[t] @ device_to_float(A[p][s]).astype(np.float64)) @ device_to_float(B[p][s]).astype(np.float64)
            at += n
    return y


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (12, 3)])
def test_prompts_and_steps(torch, fmt, graph, window, sinks):
    from decode_layer import AttentionBlock
    hq, hkv, d, batch = 4, 2, 64, 4
    projs = [wl.ProjSpec("qkv", "column", 256, (hq * d, hkv * d, hkv * d)), wl.ProjSpec("o", "row", hq * d, (192,))]
    block = AttentionBlock(projs, d, batch, 80, page_size=16, fp8=fmt == "fp8", int8=fmt == "int8", window=window, sinks=sinks, norm=True,
                           positions=256, seed=7)
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda n: torch.randn((n, 256), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    prompts = [1, 17, 38, 45]
    # the prompts in two chunks; attention is checked on the cache as it is then
    w = [device_to_float(block.norms[k]).astype(np.float64) for k in ("q_norm", "k_norm")]
    cos, sin = (t.cpu().numpy().astype(np.float64) for t in (block.cos, block.sin))

    def heads(qkv, pos):
        """Normed and rotated queries."""
        x = qkv[:, :hq * d].reshape(-1, hq, d)
        return okv.rotate(okv.head_norm(x, w[0], 1e-6), cos[pos][:, None], sin[pos][:, None])

    for s, n in enumerate(prompts):
        for start, m in ((0, min(n, 20)), (20, n - 20)):
            if m <= 0:
                continue
            x = draw(m)
            out = block.prompt(s, x, s % 4, start)
            assert int(block.lens[s]) == start + m
            k, v = _held(torch, block, s, start + m)
            qkv = _project(block, 0, device_to_float(x).astype(np.float64), [s % 4] * m)
            q = heads(wl.bf16_round(qkv)[1].astype(np.float64), np.arange(start, start + m))
            attn, _, _ = okv.attend_rows(q, k, v, d ** -0.5, okv.sees(start + m, m, window, sinks))
            # (a chain of projection, norm, attention and projection: each to about 1 % of its size)
            want = _project(block, 1, attn.reshape(m, -1), [s % 4] * m)
            assert np.abs(device_to_float(out) - want).max() <= 6e-2 * np.abs(want).max(), (s, start)
    block.begin()
    step = block.step
    if graph:
        state = [block.cache.k.view(torch.uint8), block.cache.v.view(torch.uint8), block.lens, block.index, block.positions]
        if fmt == "int8":
            state.append(block.cache.scales)
        keep = [x.clone() for x in state]
        block.step()
        torch.cuda.synchronize()
        for x, y in zip(state, keep):
            x.copy_(y)
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            block.step()
        step = cg.replay
    for k_ in range(20):
        block.x.copy_(draw(batch))
        lens = block.lens.tolist()
        step()
        torch.cuda.synchronize()
        q = device_to_float(block.q.contiguous()).astype(np.float64).reshape(batch, hq, d)
        qkv = _project(block, 0, device_to_float(block.x).astype(np.float64), block.ids.tolist())
        rot = heads(qkv, np.array(lens))
        assert np.abs(q - rot).max() <= 2e-2 * max(1.0, np.abs(rot).max())
        attn = device_to_float(block.attn).astype(np.float64).reshape(batch, hq, d)
        for b in range(batch):
            n = lens[b] + 1
            k, v = _held(torch, block, b, n)
            _attention(q[b:b + 1], k, v, okv.sees(n, 1, window, sinks), attn[b:b + 1], (k_, b))
            # the new value: the projection's, as the format holds it
            vrow = device_to_float(block.qkv_out).astype(np.float64)[b, (hq + hkv) * d:].reshape(hkv, d)
            if fmt == "fp8":
                vrow = np.clip(vrow, -448 * 0.02, 448 * 0.02)
            top = np.abs(v[:, (n - 1) // 16 * 16:]).max(axis=(1, 2))[:, None]
            tol = {"bf16": 0, "fp8": 2.0 ** -4 * np.abs(vrow) * 1.07 + 2.0 ** -10 * 0.02, "int8": top / 127 * 0.51 + 2.0 ** -8 * (np.abs(vrow) + top / 127)}[fmt]
            assert (np.abs(v[:, n - 1] - vrow) <= tol).all(), (k_, b)
        out = device_to_float(block.out)
        assert bdlora.rel_errors(out, _project(block, 1, attn.reshape(batch, -1), block.ids.tolist()))["pointwise"] <= 1e-2
    assert block.lens.tolist() == [n + 20 for n in prompts]
    assert block.cache.device_error() == 0 and block.pool.device_error() == 0
    if graph:
        del cg, step
    block.close()


def test_two_caches_on_two_streams_and_two_graphs_of_one(torch):
    import paper_2510_23346_amd as bd
    rng = np.random.default_rng(3)
    caches, args, want = [], [], []
    n_pages, ps, T, L = 200, 16, 160, 700
    table = _i32(torch, np.arange(4 * 45).reshape(4, 45))
    lens, begin = _i32(torch, [L, 3, 640, 50]), _i32(torch, [0, 100, 101, 150, 160])
    bits, _ = wl.bf16_round(rng.standard_normal((T, 8 * 128)) * 2)
    q = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    lens2, q4 = _i32(torch, [L, 3, 640, 50]), q[:4].clone()
    for seed in range(2):
        c = bd.KVCache(8, 1, 128, n_pages, ps, 4, fmt=bd.KV_INT8)
        g = torch.Generator(device="cuda").manual_seed(seed)
        c.k.copy_(torch.randint(-127, 128, c.k.shape, generator=g, device="cuda").to(torch.int8))
        c.v.copy_(torch.randint(-127, 128, c.v.shape, generator=g, device="cuda").to(torch.int8))
        c.scales.copy_(torch.rand(c.scales.shape, generator=g, device="cuda") / 100 + 0.001)
        caches.append(c)
        args.append((torch.zeros_like(q), torch.zeros_like(q4)))
        c.attend_prompt(q, begin, table, lens, args[-1][0], window=300, sinks=5)
        c.attend(q4, table, lens2, args[-1][1])
        torch.cuda.synchronize()
        want.append([t.clone() for t in args[-1]])
    assert not torch.equal(want[0][0], want[1][0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(10):
        for c, a, s in zip(caches, args, streams):
            c.attend_prompt(q, begin, table, lens, a[0], window=300, sinks=5, stream=s)
            c.attend(q4, table, lens2, a[1], stream=s)
        torch.cuda.synchronize()
        for a, w in zip(args, want):
            assert torch.equal(a[0], w[0]) and torch.equal(a[1], w[1])
            a[0].zero_(), a[1].zero_()
    # two graphs of one cache share its workspace, replayed one after the other beside eager calls
    graphs = []
    for f in (lambda: caches[0].attend_prompt(q, begin, table, lens, args[0][0], window=300, sinks=5),
              lambda: caches[0].attend(q4, table, lens2, args[0][1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    other = torch.zeros_like(q)
    for turn in range(6):
        args[0][0].zero_(), args[0][1].zero_(), other.zero_()
        graphs[turn % 2].replay()
        caches[0].attend_prompt(q, begin, table, lens, other, window=300, sinks=5)
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(args[0][0], want[0][0]) and torch.equal(args[0][1], want[0][1]) and torch.equal(other, want[0][0])
    del graphs, g
    for c in caches:
        assert c.device_error() == 0
        c.close()


def test_a_prompt_row_by_row_is_the_single_token_call(torch):
    # the same rows through attend_prompt and attend: they differ by the roundings of the probabilities
    import paper_2510_23346_amd as bd
    n, T = 1500, 40
    for fmt in (bd.KV_BF16, bd.KV_INT8):
        c = bd.KVCache(8, 2, 128, 100, 16, T, fmt=fmt)
        g = torch.Generator(device="cuda").manual_seed(1)
        if fmt == bd.KV_INT8:
            c.k.copy_(torch.randint(-127, 128, c.k.shape, generator=g, device="cuda").to(torch.int8))
            c.v.copy_(torch.randint(-127, 128, c.v.shape, generator=g, device="cuda").to(torch.int8))
            c.scales.copy_(torch.rand(c.scales.shape, generator=g, device="cuda") / 60 + 0.001)
        else:
            c.k.copy_(torch.randn(c.k.shape, generator=g, device="cuda"))
            c.v.copy_(torch.randn(c.v.shape, generator=g, device="cuda"))
        table = torch.randperm(100, generator=g, device="cuda").to(torch.int32)[None]
        q = torch.randn((T, 1024), generator=g, device="cuda").to(torch.bfloat16)
        a, b = torch.zeros_like(q), torch.zeros_like(q)
        la, lb = (torch.zeros((T, 8), device="cuda") for _ in range(2))
        for window, sinks in ((0, 0), (700, 0), (700, 33)):
            c.attend_prompt(q, _i32(torch, [0, T]), table, _i32(torch, [n]), a, window=window, sinks=sinks, lse=la)
            own = np.arange(n - T, n)
            starts = _i32(torch, own - window + 1) if window else None
            c.attend(q, table.expand(T, -1).contiguous(), _i32(torch, own + 1), b, starts=starts, sinks=sinks, lse=lb)
            x, y = device_to_float(a).astype(np.float64), device_to_float(b).astype(np.float64)
            # out: 2^-8 of each for its own rounding, 2^-8 sum p |v| <= 2^-8 of the largest value
            top = (c.v.float() * (c.scales[..., 1].repeat_interleave(16, 2)[..., None] if fmt == bd.KV_INT8 else 1.0)).abs().max().item()
            assert (np.abs(x - y) <= 2.0 ** -7 * np.abs(y) + 2.0 ** -8 * top).all()
            assert (la - lb).abs().max().item() <= 2.0 ** -16
        c.close()
