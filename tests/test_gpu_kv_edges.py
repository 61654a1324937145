"""Attention where a number of the cache is a zero scale: attend and attend_prompt
give what the formula gives.  Tolerances as in
test_gpu_kv_prompt.py."""
import numpy as np
import pytest

from oracle import kv as okv
from test_gpu_kv_prompt import _compare, _i32, _queries, torch  # noqa: F401  (torch: a fixture)
from workloads.gpu import device_to_float
from workloads.kv import DrawnCache

pytestmark = pytest.mark.gpu


def _scales(dc, b, which, blocks, value):
    """Give blocks of sequence b of an int8 cache (of keys: which 0, of values: 1) another scale."""
    page, place = dc.where(b)
    plain = (dc.k, dc.v)[which][b]
    stored = dc.take((dc.K, dc.V)[which], b, plain.shape[1])
    for x in blocks:
        at = slice(16 * x, min(16 * x + 16, plain.shape[1]))
        dc.S[page[at], :, place[at] // 16, which] = value
        plain[:, at] = stored[:, at] * np.float64(np.float32(value))


# ------------------------------------------------ scales of 0 (int8)

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq", [4, 20])
@pytest.mark.parametrize("value", [0.0, 2.0 ** -64 / 127])
@pytest.mark.parametrize("scale", [None, 0.0])
def test_single_tokens_over_blocks_of_scale_zero(torch, d, hq, value, scale):  # noqa: F811
    # the blocks that len, starts and sinks cut through, and a whole one; two entries of nothing
    lens, starts = [1, 5, 21, 40, 100, 300, 777], [0, 0, 3, 37, 70, 150, 700]
    dc = DrawnCache(lens, 1, d, 16, seed=d, int8=True)
    for b, (n, s) in enumerate(zip(lens, starts)):
        for which in (0, 1):
            _scales(dc, b, which, {0, s // 16, (n - 1) // 16, n // 32}, value)
    cache, table, dl = dc.device(n_q_heads=hq)
    q, x = _queries(torch, len(lens), hq, d, 1)
    for sinks, begin in ((0, None), (0, starts), (2, starts), (37, starts)):
        out, lse = torch.empty_like(q), torch.empty((len(lens), hq), device="cuda")
        cache.attend(q, table, dl, out, starts=begin and _i32(torch, begin), lse=lse, sinks=sinks, scale=scale)
        o, z = device_to_float(out).astype(np.float64).reshape(-1, 1, hq, d), lse.cpu().numpy()
        for b, n in enumerate(lens):
            j = np.arange(n)
            seen = ((j >= (begin[b] if begin else 0)) | (j < sinks))[None, :]
            _compare(o[b], z[b:b + 1], x[b:b + 1], dc.k[b], dc.v[b], d ** -0.5 if scale is None else scale, seen, 15, (sinks, b))
    assert cache.device_error() == 0
    cache.close()


@pytest.mark.parametrize("value", [0.0, 2.0 ** -64 / 127])
@pytest.mark.parametrize("new", [[1, 2, 3, 7], [40, 70, 1, 130]])
def test_prompts_over_blocks_of_scale_zero(torch, new, value):  # noqa: F811
    lens = [41, 90, 21, 333]
    dc = DrawnCache(lens, 1, 128, 64, seed=len(new), int8=True)
    for b, n in enumerate(lens):
        for which in (0, 1):
            _scales(dc, b, which, {0, (n - 1) // 16, n // 32, (n - new[b]) // 16}, value)
    cache, table, dl = dc.device(n_q_heads=4)
    begin = np.concatenate([[0], np.cumsum(new)])
    q, x = _queries(torch, begin[-1], 4, 128, 1)
    for window, sinks, scale in ((0, 0, None), (19, 3, None), (50, 20, 0.0)):
        out, lse = torch.empty_like(q), torch.empty((begin[-1], 4), device="cuda")
        cache.attend_prompt(q, _i32(torch, begin), table, dl, out, window=window, sinks=sinks, scale=scale, lse=lse)
        o, z = device_to_float(out).astype(np.float64).reshape(-1, 4, 128), lse.cpu().numpy()
        for b, n in enumerate(lens):
            r = slice(begin[b], begin[b + 1])
            _compare(o[r], z[r], x[r], dc.k[b], dc.v[b], 128 ** -0.5 if scale is None else scale, okv.sees(n, new[b], window, sinks), 8,
                     (window, b))
    cache.close()


def test_single_tokens_over_a_cache_that_holds_nothing_yet(torch):  # noqa: F811
    # as allocated: all entries 0, so the mean of the values is 0 and the sum of exponentials their number
    import paper_2510_23346_amd as bd
    cache = bd.KVCache(4, 1, 128, 3, 16, 4, fmt=bd.KV_INT8)
    table, lens = torch.zeros((4, 3), dtype=torch.int32, device="cuda"), _i32(torch, [1, 16, 33, 0])
    q, _ = _queries(torch, 4, 4, 128, 1)
    out, lse = torch.full_like(q, 7.0), torch.empty((4, 4), device="cuda")
    cache.attend(q, table, lens, out, lse=lse)
    assert not out.any()
    assert np.allclose(lse.cpu().numpy(), np.array([0, np.log(16), np.log(33), -np.inf])[:, None], atol=2.0 ** -19)
    cache.close()
