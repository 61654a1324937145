"""Drawn key-value caches for the tests and the example: values, pages, page
tables.  No arithmetic of the operators happens here.

Everything that no call may read holds NaN (places behind a sequence's length,
pages of no sequence) or a page number that does not exist (places of the
page table behind a sequence's last page)."""
from __future__ import annotations

import numpy as np

from . import bf16_bits_to_float, bf16_round


class DrawnCache:
    """``lens[b]`` entries per sequence, in pages of ``page_size`` in random
    order.  ``k[b]``, ``v[b]``: float64 ``[n_kv_heads, len, head_dim]``, the
    stored values (an 8-bit cache: times their scale); ``weight[b]``,
    ``pos[b]``.  ``spare`` pages belong to no sequence, ``room[b]`` more
    entries have pages already (``room``: int or per sequence).  ``int8``: a
    cache with a scale for each block of 16 entries (``S``), drawn log-normal."""

    def __init__(self, lens, n_kv_heads, head_dim, page_size, seed, fp8=False, k_scale=1.0, v_scale=1.0, spare=2, room=0,
                 wide=2, int8=False):
        from oracle.kv import e4m3_encode, e4m3_values
        rng = np.random.default_rng([seed, 11])
        self.lens = np.asarray(lens, np.int32)
        self.int8 = int8
        self.fp8, self.ps, self.hkv, self.d = fp8, page_size, n_kv_heads, head_dim
        self.scales = (k_scale, v_scale)
        B = len(self.lens)
        rooms = np.broadcast_to(np.asarray(room), (B,))
        need = -(-(self.lens + rooms) // page_size)
        self.n_pages = int(need.sum()) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((B, max(1, int(need.max()) if B else 1) + wide), -7, np.int32)
        self.table[:, 1::2] = 2 ** 31 - 1
        at = 0
        for b in range(B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        shape = (self.n_pages, n_kv_heads, page_size)
        nan = 0x7F if int8 else 0xFF if fp8 else 0x7FFF
        self.K, self.V = (np.full(shape + (head_dim,), nan, np.int8 if int8 else np.uint8 if fp8 else np.uint16) for _ in range(2))
        self.S = np.full(shape[:2] + (page_size // 16, 2), np.nan, np.float32) if int8 else None
        self.W = np.full(shape, np.nan, np.float32)
        self.P = np.full(shape, 2 ** 31 - 1, np.int32)
        self.k, self.v, self.weight, self.pos = [], [], [], []
        values = e4m3_values()
        for b, n in enumerate(self.lens):
            for stored, plain, scale in ((self.K, self.k, k_scale), (self.V, self.v, v_scale)):
                x = rng.standard_normal((n_kv_heads, n, head_dim))
                if int8:
                    bits = rng.integers(-127, 128, (n_kv_heads, n, head_dim)).astype(np.int8)
                    f = np.exp(0.3 * rng.standard_normal((n_kv_heads, -(-n // 16)))).astype(np.float32) / np.float32(127)
                    plain.append(bits * np.repeat(f, 16, 1)[:, :n, None].astype(np.float64))
                    page, place = self.where(b, n)
                    self.S[page[::16], :, place[::16] // 16, 0 if stored is self.K else 1] = f.T
                elif fp8:
                    bits = e4m3_encode(x / scale)
                    plain.append(values[bits] * np.float64(np.float32(scale)))
                else:
                    bits = bf16_round(x)[0]
                    plain.append(bf16_bits_to_float(bits).astype(np.float64))
                self.put(stored, b, bits)
            w = np.exp(rng.standard_normal((n_kv_heads, n))).astype(np.float32)
            p = np.stack([np.sort(rng.choice(2 * n, n, replace=False)) if n else np.zeros(0) for _ in range(n_kv_heads)])
            self.weight.append(w)
            self.pos.append(p.astype(np.int32))
            self.put(self.W, b, w)
            self.put(self.P, b, self.pos[b])

    def where(self, b, n=None):
        """(pages, places) of the first n entries of sequence b."""
        i = np.arange(self.lens[b] if n is None else n)
        return self.table[b, i // self.ps], i % self.ps

    def put(self, pages, b, rows):
        """rows [heads, n, ...] into the pages of sequence b."""
        p, s = self.where(b, rows.shape[1])
        pages[p, :, s] = np.swapaxes(rows, 0, 1)

    def take(self, pages, b, n):
        """The first n entries of sequence b: [heads, n, ...]."""
        p, s = self.where(b, n)
        return np.swapaxes(pages[p, :, s], 0, 1)

    def device(self, weights=True, n_q_heads=None, max_seqs=None, **kw):
        """(KVCache over device copies of the pages, device page table, lens)."""
        import torch

        import paper_2510_23346_amd as bd
        kind = torch.int8 if self.int8 else torch.float8_e4m3fn if self.fp8 else torch.bfloat16
        dt = np.int8 if self.int8 else np.uint8 if self.fp8 else np.int16
        k, v = (torch.from_numpy(x.view(dt).copy()).cuda().view(kind) for x in (self.K, self.V))
        if self.int8:
            weights = False
            kw["scales"] = torch.from_numpy(self.S.copy()).cuda()
        cache = bd.KVCache(n_q_heads or self.hkv, self.hkv, self.d, self.n_pages, self.ps, max_seqs or max(1, len(self.lens)),
                           fmt=bd.KV_INT8 if self.int8 else bd.KV_FP8_E4M3 if self.fp8 else bd.KV_BF16, k_scale=self.scales[0], v_scale=self.scales[1], k=k,
                           v=v, weight=torch.from_numpy(self.W.copy()).cuda() if weights else None,
                           pos=torch.from_numpy(self.P.copy()).cuda() if weights else None, **kw)
        return cache, torch.from_numpy(self.table.copy()).cuda(), torch.from_numpy(self.lens.copy()).cuda()


def host_bits(t) -> np.ndarray:
    """A bf16 or 8-bit device tensor's bit patterns."""
    import torch
    if t.element_size() == 1:
        return t.detach().contiguous().view(torch.uint8).cpu().numpy()
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
