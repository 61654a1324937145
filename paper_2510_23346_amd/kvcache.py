"""The key-value cache of one decoder layer on one shard (``bdlora_kv_*``).

:class:`KVCache` stands between the qkv and the o projection of a layer:
``append`` rotates the new tokens' queries and keys and stores keys and
values, ``attend`` is the attention of one new token per sequence, ``evict``
cuts sequences to a budget by the attention their entries got.  As in the rest
of the binding, only arguments are checked and marshalled here.
"""
from __future__ import annotations

import ctypes as _c
import math
from typing import Tuple

from . import KV_BF16, KV_FP8_E4M3, KVDesc, _check, lib

__all__ = ["KVCache", "kv_bytes"]


def _int32(name: str, v) -> int:
    """``v`` as the C ABI's int32 takes it (ctypes would cut it to 32 bits)."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name} = {v} does not fit 32 bits")
    return v


def _desc(n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, fmt, k_scale=1.0, v_scale=1.0) -> KVDesc:
    return KVDesc(_int32("n_q_heads", n_q_heads), _int32("n_kv_heads", n_kv_heads), _int32("head_dim", head_dim),
                  _int32("page_size", page_size), _int32("n_pages", n_pages), _int32("max_seqs", max_seqs), _int32("fmt", fmt),
                  float(k_scale), float(v_scale))


def kv_bytes(n_q_heads: int, n_kv_heads: int, head_dim: int, page_size: int, n_pages: int, max_seqs: int, *,
             fmt: int = KV_BF16, weights: bool = False) -> Tuple[int, int]:
    """Bytes of one page (k and v; with ``weights`` weight and pos too) and of
    a cache's workspace (pure host)."""
    d = _desc(n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, fmt)
    a, b = _c.c_int64(), _c.c_int64()
    _check(lib().bdlora_kv_bytes(_c.byref(d), int(weights), _c.byref(a), _c.byref(b)))
    return a.value, b.value


class KVCache:
    """A paged key-value cache.

    ``k`` and ``v`` are device tensors ``[n_pages, n_kv_heads, page_size,
    head_dim]`` (bf16, or ``torch.float8_e4m3fn`` standing for ``k_scale`` or
    ``v_scale`` times their values), ``weight`` (fp32) and ``pos`` (int32)
    ``[n_pages, n_kv_heads, page_size]``.  They are allocated (zeroed) where
    they are not given; weight and pos only with ``weights=True``, and a cache
    without them cannot accumulate or evict.

    ``table`` arguments are int32 device tensors ``[sequences, width]``:
    entry i of a sequence lies in place ``i % page_size`` of page ``table[row,
    i // page_size]``.  Calls enqueue on ``stream`` (the current one).
    """

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, page_size: int, max_seqs: int, *,
                 fmt: int = KV_BF16, k_scale: float = 1.0, v_scale: float = 1.0, weights: bool = False, device: int = 0,
                 k=None, v=None, weight=None, pos=None):
        import torch
        self._h = None
        d = _desc(n_q_heads, n_kv_heads, head_dim, page_size, n_pages, max_seqs, fmt, k_scale, v_scale)
        self.n_q_heads, self.n_kv_heads, self.head_dim = d.n_q_heads, d.n_kv_heads, d.head_dim
        self.n_pages, self.page_size, self.max_seqs, self.fmt = d.n_pages, d.page_size, d.max_seqs, d.format
        self.device = _int32("device", device)
        _check(lib().bdlora_kv_bytes(_c.byref(d), 0, None, None))       # refuses a bad description before any allocation
        self._bf16, self._i32, self._f32 = torch.bfloat16, torch.int32, torch.float32
        shape = (self.n_pages, self.n_kv_heads, self.page_size)
        kind = torch.float8_e4m3fn if self.fmt == KV_FP8_E4M3 else torch.bfloat16
        weights = weights or weight is not None or pos is not None

        def buffer(name, t, shape, kind):
            if t is None:
                return torch.zeros(shape, dtype=kind, device=f"cuda:{self.device}")
            if tuple(t.shape) != shape or t.dtype != kind or not t.is_contiguous() or t.get_device() != self.device:
                raise ValueError(f"{name} must be a contiguous {kind} tensor {shape} on cuda:{self.device}")
            return t

        self.k = buffer("k", k, shape + (self.head_dim,), kind)
        self.v = buffer("v", v, shape + (self.head_dim,), kind)
        self.weight = buffer("weight", weight, shape, torch.float32) if weights else None
        self.pos = buffer("pos", pos, shape, torch.int32) if weights else None
        h = _c.c_void_p()
        _check(lib().bdlora_kv_create(_c.byref(d), self.k.data_ptr(), self.v.data_ptr(),
                                      self.weight.data_ptr() if weights else None, self.pos.data_ptr() if weights else None,
                                      self.device, _c.byref(h)))
        self._h = h
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda device: torch.cuda.current_stream(device).cuda_stream)
        self._scale = 1.0 / math.sqrt(self.head_dim)
        self._qw = self.n_q_heads * self.head_dim
        self._qkvw = self._qw + 2 * self.n_kv_heads * self.head_dim
        L = lib()
        self._append, self._attend, self._evict = L.bdlora_kv_append, L.bdlora_kv_attend, L.bdlora_kv_evict

    # -- lifetime ---------------------------------------------------------
    def close(self):
        if getattr(self, "_h", None):
            _check(lib().bdlora_kv_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- arguments --------------------------------------------------------
    # (these checks run in front of every call, and a call's kernel may take 5
    # us: they touch each property of a tensor once)
    def _stream(self, stream):
        if stream is None:
            # the handle alone: torch.cuda.current_stream() builds an object
            # around it, which takes 2.7 us
            return self._raw_stream(self.device)
        return stream if isinstance(stream, int) else int(stream.cuda_stream)

    def _rows(self, name, t, n, width):
        """Row stride of a bf16 tensor of n rows: [n, width], or [n, heads, head_dim]."""
        sh, st = t.shape, t.stride()
        if t.dtype is self._bf16 and t.get_device() == self.device:
            if sh == (n, width):
                if st[1] == 1:
                    return st[0] if n > 1 else width
            elif len(sh) == 3 and sh == (n, width // self.head_dim, self.head_dim) and st[2] == 1 and \
                    (st[1] == self.head_dim or sh[1] == 1):
                return st[0] if n > 1 else width
        raise ValueError(f"{name} must be a bf16 tensor [{n}, {width}] on cuda:{self.device} with contiguous rows")

    def _ints(self, name, t, n):
        if t.dtype is self._i32 and t.shape == (n,) and t.get_device() == self.device and t.is_contiguous():
            return t.data_ptr()
        raise ValueError(f"{name} must be a contiguous int32 tensor of {n} values on cuda:{self.device}")

    def _table(self, t):
        sh, st = t.shape, t.stride()
        if t.dtype is self._i32 and len(sh) == 2 and (st[1] == 1 or sh[1] <= 1) and t.get_device() == self.device:
            return t.data_ptr(), (st[0] if sh[0] > 1 else sh[1]), sh[1], sh[0]
        raise ValueError(f"table must be an int32 tensor [sequences, width] on cuda:{self.device} with contiguous rows")

    def _floats(self, name, t, shape):
        if t.dtype is self._f32 and t.shape == shape and t.get_device() == self.device and t.is_contiguous():
            return t.data_ptr()
        raise ValueError(f"{name} must be a contiguous fp32 tensor {list(shape)} on cuda:{self.device}")

    # -- operators --------------------------------------------------------
    def append(self, qkv, cos, sin, seqs, index, positions, table, lens, q_out, interleaved: bool = False, stream=None):
        """Rotate the queries and keys of ``qkv [T, (n_q_heads + 2
        n_kv_heads) head_dim]`` (the qkv projection's output), store keys and
        values as entries ``index`` of table rows ``seqs`` (-1: not stored),
        raise ``lens`` (may be None; not the memory of the other integers,
        which are still read while it changes) to cover them, and write the
        rotated queries to ``q_out`` (it may be qkv's own query columns).
        ``cos`` and ``sin``: fp32 ``[positions, head_dim / 2]``."""
        T = qkv.shape[0]
        qs = self._rows("qkv", qkv, T, self._qkvw)
        os_ = self._rows("q_out", q_out, T, self._qw)
        P = cos.shape[0]
        angles = (P, self.head_dim // 2)
        tp, ts, tw, n = self._table(table)
        ps, pi, pp = self._ints("seqs", seqs, T), self._ints("index", index, T), self._ints("positions", positions, T)
        pl = None
        if lens is not None:
            pl = self._ints("lens", lens, n)
            end, size = pl + 4 * n, 4 * T
            if (pl < ps + size and ps < end) or (pl < pi + size and pi < end) or (pl < pp + size and pp < end):
                raise ValueError("lens must not share memory with seqs, index or positions")
        rc = self._append(self._h, qkv.data_ptr(), qs, self._floats("cos", cos, angles), self._floats("sin", sin, angles), P,
                          int(interleaved), ps, pi, pp, T, tp, ts, tw, n, pl, q_out.data_ptr(), os_, self._stream(stream))
        if rc:
            _check(rc)

    def attend(self, q, table, lens, out, starts=None, scale=None, lse=None, accumulate: bool = False, stream=None):
        """Attention of row b of ``q [B, n_q_heads head_dim]`` over entries
        ``starts[b]`` (0) to ``lens[b]`` of table row b, into ``out`` (not
        q's memory: several workgroups read a query); ``scale`` defaults to
        ``head_dim ** -0.5``.  ``lse``: fp32 ``[B, n_q_heads]``, receives the
        log of the sum of the scores' exponentials.  ``accumulate`` adds the
        entries' probabilities to ``weight``."""
        B = q.shape[0]
        qs = self._rows("q", q, B, self._qw)
        os_ = self._rows("out", out, B, self._qw)
        tp, ts, tw, n = self._table(table)
        if n < B:
            raise ValueError(f"table has {n} rows for {B} sequences")
        qp, op = q.data_ptr(), out.data_ptr()
        if qp == op and B:
            raise ValueError("out must not be q's memory")
        rc = self._attend(self._h, qp, qs, B, tp, ts, tw, self._ints("lens", lens, B),
                          None if starts is None else self._ints("starts", starts, B),
                          self._scale if scale is None else scale, int(accumulate), op, os_,
                          None if lse is None else self._floats("lse", lse, (B, self.n_q_heads)), self._stream(stream))
        if rc:
            _check(rc)

    def evict(self, table, lens, budget: int, recent: int = 0, stream=None):
        """Cut the sequences of ``table`` to ``budget`` entries per kv head:
        the last ``recent`` positions stay, then the largest weights; kept
        entries from behind the budget move into the freed places."""
        tp, ts, tw, B = self._table(table)
        rc = self._evict(self._h, B, tp, ts, tw, self._ints("lens", lens, B), _int32("budget", budget),
                         _int32("recent", recent), self._stream(stream))
        if rc:
            _check(rc)

    def device_error(self, stream=None) -> int:
        f = _c.c_int32(0)
        _check(lib().bdlora_kv_get_device_error(self._h, self._stream(stream), _c.byref(f)))
        return f.value
