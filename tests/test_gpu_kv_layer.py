"""The attention block of examples/decode_layer.py: projections with adapters,
cache entry, attention and eviction together, step after step, every stage
against the float64 oracle on what the stage before it left."""
import os
import sys

import numpy as np
import pytest

import workloads as wl
from oracle import bdlora, kv as okv
from workloads.gpu import device_to_float
from workloads.kv import host_bits

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    import paper_2510_23346_amd as bd
    bd.lib()
    return torch


def _entries(block, what, b, n):
    """[heads, n, ...] of sequence b."""
    t = block.table.cpu().numpy()
    i = np.arange(n)
    ps = block.cache.page_size
    return np.swapaxes(what[t[b, i // ps], :, i % ps], 0, 1)


def _stored(block, bits, scale):
    if bits.dtype == np.uint8:
        return okv.e4m3_values()[bits] * np.float64(np.float32(scale))
    return wl.bf16_bits_to_float(bits).astype(np.float64)


def _projection(block, p, x, ids):
    """Float64 of x W^T + 2 (x A) B per token."""
    w = device_to_float(block.w[p]).astype(np.float64)
    y = x @ w.T
    for t, a in enumerate(ids):
        A, B = block.adapters[a]
        at = 0
        for s, n in enumerate((block.qkv, block.o)[p].slices):
            y[t, at:at + n] += 2.0 * (x[t] @ device_to_float(A[p][s]).astype(np.float64)) @ \
                device_to_float(B[p][s]).astype(np.float64)
            at += n
    return y


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_an_attention_block(torch, fp8, graph):
    from decode_layer import AttentionBlock
    hq, hkv, d, batch, budget, recent = 4, 2, 64, 5, 40, 8
    projs = [wl.ProjSpec("qkv", "column", 256, (hq * d, hkv * d, hkv * d)), wl.ProjSpec("o", "row", hq * d, (192,))]
    block = AttentionBlock(projs, d, batch, 64, page_size=16, budget=budget, recent=recent, fp8=fp8, positions=256, seed=3)
    scale = 0.02 if fp8 else 1.0
    g = torch.Generator(device="cuda").manual_seed(5)
    prompts = [1, 17, 38, 39, 40]                # the last three pass the budget within the steps
    for s, n in enumerate(prompts):
        block.prompt(s, torch.randn((n, 256), generator=g, device="cuda").to(torch.bfloat16), s % 4)
    block.begin()
    assert block.lens.tolist() == prompts
    ids = block.ids.tolist()
    step = block.step
    if graph:
        state = [block.cache.k.view(torch.uint8), block.cache.v.view(torch.uint8), block.cache.weight, block.cache.pos, block.lens,
                 block.index, block.positions]
        keep = [x.clone() for x in state]
        block.step()                             # warm up
        torch.cuda.synchronize()
        for x, y in zip(state, keep):
            x.copy_(y)
        cg = torch.cuda.CUDAGraph()
        with torch.cuda.graph(cg):
            block.step()
        step = cg.replay
    for k in range(6):
        block.x.copy_(torch.randn(block.x.shape, generator=g, device="cuda"))
        lens, pos = block.lens.tolist(), block.positions.tolist()
        W0, P0 = block.cache.weight.cpu().numpy(), block.cache.pos.cpu().numpy()
        K0 = host_bits(block.cache.k)
        step()
        torch.cuda.synchronize()
        # o's input and output, and qkv's keys and values (its queries were rotated in place)
        x = device_to_float(block.x).astype(np.float64)
        qkv = _projection(block, 0, x, ids)
        attn = device_to_float(block.attn).astype(np.float64)
        assert bdlora.rel_errors(device_to_float(block.out), _projection(block, 1, attn, ids))["pointwise"] <= 1e-2
        got = device_to_float(block.qkv_out).astype(np.float64)
        assert bdlora.rel_errors(got[:, hq * d:], qkv[:, hq * d:])["pointwise"] <= 1e-2
        cos, sin = (t.cpu().numpy().astype(np.float64) for t in (block.cos, block.sin))
        q = got[:, :hq * d].reshape(batch, hq, d)
        for b in range(batch):
            rot = okv.rotate(qkv[b, :hq * d].reshape(hq, d), cos[pos[b]], sin[pos[b]])
            assert np.abs(q[b] - rot).max() <= 2e-2 * max(1.0, np.abs(rot).max())
        # the new entry, and with it the cache that attention read
        assert block.positions.tolist() == [p + 1 for p in pos]
        W1, P1 = block.cache.weight.cpu().numpy(), block.cache.pos.cpu().numpy()
        K1 = host_bits(block.cache.k)
        for b in range(batch):
            n = lens[b] + 1
            krow = got[b, hq * d:(hq + hkv) * d].reshape(hkv, d)
            vrow = got[b, (hq + hkv) * d:].reshape(hkv, d)
            rot = okv.rotate(krow, cos[pos[b]], sin[pos[b]])
            keys = _stored(block, _entries(block, K0, b, n), scale)
            new = okv.e4m3_values()[okv.e4m3_encode(rot / scale)] * scale if fp8 else rot
            keys[:, n - 1] = new
            w = _entries(block, W0, b, n).astype(np.float64)
            w[:, n - 1] = 0
            p = _entries(block, P0, b, n)
            p[:, n - 1] = pos[b]
            _, _, share = okv.attend(q[b], keys, np.zeros_like(keys), d ** -0.5)
            w += share
            # eviction: by the weights (within what the sums may be off, ties are not expected)
            m = min(n, budget)
            assert block.lens.tolist()[b] == m
            for h in range(hkv):
                places, sources = okv.evict_plan(w[h], p[h], budget, recent)
                order = np.arange(n)
                order[places] = sources
                assert np.array_equal(_entries(block, P1, b, m)[h], p[h][order[:m]]), (k, b, h)
                assert np.allclose(_entries(block, W1, b, m)[h], w[h][order[:m]], rtol=2e-2, atol=1e-3)
                # (8 bits: at most a step from the oracle's, where the rotation's
                # last bits decide a tie; bf16: half a step from its 64 bits)
                want = keys[h][order[:m]]
                step_ = 2.0 ** -3 * np.abs(want) + 2.0 ** -9 * scale if fp8 else 2.0 ** -8 * np.abs(want) + 2.0 ** -20
                assert (np.abs(_stored(block, _entries(block, K1, b, m)[h], scale) - want) <= 1.001 * step_).all()
            if n <= budget:                      # (nothing moved: the values are those that attention read)
                vals = _stored(block, _entries(block, host_bits(block.cache.v), b, n), scale)
                # (values are not rotated: exactly the oracle's rounding of them)
                inv = np.float32(1) / np.float32(scale)
                want = okv.e4m3_values()[okv.e4m3_encode(vrow.astype(np.float32) * inv)] * np.float64(np.float32(scale)) if fp8 else vrow
                assert np.array_equal(vals[:, n - 1], want)
                ref, _, _ = okv.attend(q[b], _stored(block, _entries(block, K1, b, n), scale), vals, d ** -0.5)
                assert np.abs(attn[b].reshape(hq, d) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-3
    assert block.cache.device_error() == 0 and block.pool.device_error() == 0
    assert block.lens.tolist() == [min(budget, n + 6) for n in prompts]
    block.close()
