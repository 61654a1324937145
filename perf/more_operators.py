"""Further operators of the key-value cache, as measurable cases.

All work on the paged cache of one decoder layer on one tensor-parallel shard
(pages [n_pages, n_kv_heads, page_size, head_dim]):

attend  attention of one new token per sequence, over an 8-bit cache with a
        scale for each block of 16 entries of a head, and over a sliding window
        beside a few first entries that stay visible (sinks), in any format;
prompt  attention of many new tokens of each sequence (a prompt, a chunk of
        one, drafted tokens, single tokens among them), causal, over the
        cache, with window and sinks;
append  norms of queries and keys for each head and their rotation in one
        pass, with the entry of keys and values into the cache;
store   the same into the block-scaled 8-bit cache, quantised as it is
        written, and the blocks that were written read back;
read    whole sequences of such a cache read back.

Head counts are those of the Llama shards in ``workloads/`` (tensor-parallel
degree 8, 4 and 1), batch sizes and prompt lengths those of its workloads;
sequences hold up to 131072 entries.

Cached keys and values are N(0, 1), queries N(0, 4), so that the scores of a
sequence have a standard deviation of 2 and a few entries matter.  In the
8-bit cache each block has a size of its own, log-normal.  Pages lie in random
order; page 0 is the null page that a page table's unused places name.
"""
import math

import numpy as np
import torch

own = False

FP8_K, FP8_V = 0.015, 0.0125     # scales of an e4m3 cache
POSITIONS = 16384                # rows of the rotary tables
BLOCK = 16                       # entries of a head that share a scale
LEAST = 2.0 ** -64               # a block's largest magnitude counts as no less
EPS = 1e-6
HEADS = {"1b/4": (8, 2, 64), "8b/8": (4, 1, 128), "8b/4": (8, 2, 128), "8b/1": (32, 8, 128), "70b/8": (8, 1, 128),
         "70b/4": (16, 2, 128)}                           # query heads, kv heads, head size of a shard


def _attend(name, shard, B, length, lens="same", *, page=16, fmt="bf16", window=0, sinks=0, empty=0):
    """lens: "same" (all `length`), "spread" (even from length / 16) or "log"
    (even in the logarithm, from 1).  window: only the last so many entries
    are attended to (0: all), and the first `sinks`.  empty: so many sequences
    have no entry yet."""
    return {"name": name, "op": "attend", "shard": shard, "B": B, "len": length, "lens": lens, "page": page, "fmt": fmt,
            "window": window, "sinks": sinks, "empty": empty}


def _prompt(name, shard, prompts, prompt, decode, length, *, page=64, fmt="bf16", window=0, sinks=0):
    """`prompts` sequences with `prompt` new tokens each and `decode` with one,
    behind up to `length` entries that are there already."""
    return {"name": name, "op": "prompt", "shard": shard, "prompts": prompts, "prompt": prompt, "decode": decode,
            "len": length, "page": page, "fmt": fmt, "window": window, "sinks": sinks}


def _append(name, shard, prompts, prompt, decode, length, *, page=16, fmt="bf16", norm=True, interleaved=False):
    """`prompts` runs of `prompt` tokens and `decode` single tokens, whose
    sequences hold up to `length` entries."""
    return {"name": name, "op": "store" if fmt == "int8" else "append", "shard": shard, "prompts": prompts, "prompt": prompt,
            "decode": decode, "len": length, "page": page, "fmt": fmt, "norm": norm, "interleaved": interleaved}


def _read(name, shard, B, length, lens="spread", *, page=64):
    return {"name": name, "op": "read", "shard": shard, "B": B, "len": length, "lens": lens, "page": page, "fmt": "int8"}


def listed():
    return [
        # a single user early in an answer, 8-bit cache: launch and call latency
        _attend("attend-int8-8b-B1-777", "8b/8", 1, 777, fmt="int8"),
        # the usual decode batch at long context, 8-bit cache
        _attend("attend-int8-8b-B64-8192", "8b/8", 64, 8192, "spread", page=64, fmt="int8"),
        # a ragged batch of a small model (head size 64) that sees 300 entries and 4 sinks, some requests new
        _attend("attend-sinks-1b-B37-ragged", "1b/4", 37, 2048, "log", window=300, sinks=4, empty=3),
        # long streams, a window of half of them
        _attend("attend-sinks-8b-B16-32768", "8b/8", 16, 32768, page=64, window=16384, sinks=64),
        # the prompts of the prefill workload
        _prompt("prompt-8b-8x512", "8b/8", 8, 512, 0, 0),
        # continuous batching of a large model: prompts beside decode tokens, e4m3 cache
        _prompt("prompt-70b-4x1024+192-fp8", "70b/8", 4, 1024, 192, 512, page=16, fmt="fp8"),
        # one long prompt, all heads of a model on one GPU: the heaviest call here
        _prompt("prompt-8b-1x8192", "8b/1", 1, 8192, 0, 0),
        # a book through a window, with sinks
        _prompt("prompt-sinks-70b-1x16384", "70b/8", 1, 16384, 0, 0, window=4096, sinks=4),
        # five drafted tokens of each sequence against a long 8-bit cache
        _prompt("prompt-8b-64x5-4096-int8", "8b/8", 64, 5, 0, 4096, fmt="int8"),
        # a decode step's new queries, keys and values
        _append("append-norm-8b-T64", "8b/8", 0, 0, 64, 512),
        # continuous batching into the 8-bit cache, read back
        _append("store-int8-70b-4x1024+192", "70b/8", 4, 1024, 192, 512, fmt="int8"),
        # sequences taken out of the 8-bit cache
        _read("read-int8-8b-B16-32768", "8b/4", 16, 32768),
    ]


def _log(rng, a, b):
    return int(math.exp(rng.uniform(math.log(a), math.log(b + 0.999))))


def draw(rng):
    """One more case of the same ranges."""
    shard = rng.choice(list(HEADS))
    page = rng.choice([16, 16, 32, 64, 128, 256])
    hq, hkv, d = HEADS[shard]
    op = rng.choice(["attend", "attend", "prompt", "prompt", "prompt", "append", "store", "read"])
    if op == "attend":
        fmt = rng.choice(["int8", "int8", "bf16", "fp8"])
        most = 250_000_000 // (2 * hkv * d * (2 if fmt == "bf16" else 1))     # entries of all sequences together
        B = _log(rng, 1, 256)
        length = _log(rng, 1, max(1, min(131072, most // B)))
        windowed = fmt != "int8" or rng.random() < 0.4
        c = _attend("", shard, B, length, rng.choice(["same", "spread", "log"]), page=page, fmt=fmt,
                    window=_log(rng, 1, length) if windowed else 0, sinks=_log(rng, 1, 128) if windowed else 0,
                    empty=rng.randint(1, B // 4) if B >= 4 and rng.random() < 0.3 else 0)
    elif op == "prompt":
        fmt = rng.choice(["bf16", "bf16", "fp8", "int8"])
        prompts, prompt = (1, _log(rng, 1024, 12288)) if rng.random() < 0.3 else (rng.randint(1, 16), _log(rng, 2, 1024))
        decode = _log(rng, 1, 128) if rng.random() < 0.4 else 0
        length = _log(rng, 1, 8192) if rng.random() < 0.6 else 0
        # (the plain form's scores: at most 2e9 of them)
        while (prompts + decode) * prompt * hq * (length + prompt) > 2e9:
            if decode:
                decode //= 2
            elif length > 64:
                length //= 2
            elif prompts > 1:
                prompts //= 2
            else:
                prompt //= 2
        windowed = rng.random() < 0.5
        c = _prompt("", shard, prompts, prompt, decode, length, page=page, fmt=fmt,
                    window=_log(rng, 1, length + prompt) if windowed else 0, sinks=_log(rng, 1, 128) if windowed else 0)
    elif op == "read":
        B = _log(rng, 1, 64)
        c = _read("", shard, B, _log(rng, 1, min(131072, 500_000 // (B * hkv))), rng.choice(["same", "spread", "log"]), page=page)
    else:
        c = _append("", shard, 0, 0, 0, _log(rng, 1, 600), page=page, fmt="int8" if op == "store" else rng.choice(["bf16", "fp8"]),
                    norm=op == "append" or rng.random() < 0.6, interleaved=rng.random() < 0.3)
        c["decode"] = _log(rng, 1, 256) if rng.random() < 0.7 else 0
        if not c["decode"] or rng.random() < 0.5:
            c["prompts"] = rng.randint(1, 8)
            c["prompt"] = _log(rng, 1, 1024 if hkv < 8 else 256)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _lens(case):
    """The sequences' lengths, ascending (attend, read)."""
    B, top = case["B"], case["len"]
    u = (np.arange(B) + 1) / B
    if case["lens"] == "same":
        n = np.full(B, float(top))
    elif case["lens"] == "spread":
        n = top / 16 + (top - top / 16) * u
    else:
        n = np.exp(math.log(top) * u)
    n = np.maximum(1, np.rint(n)).astype(np.int64)
    n[:case.get("empty", 0)] = 0
    return n


def _counts(case):
    """Entries that are there and new tokens of each sequence (prompt, append)."""
    p, n, top = case["prompts"], case["decode"], case["len"]
    new = np.concatenate([np.full(p, case["prompt"]), np.ones(n, np.int64)]).astype(np.int64)
    if case["op"] == "prompt":
        B = p + n
        old = np.rint(top * (np.arange(B) + 1) / B).astype(np.int64)
    else:
        single = np.arange(n) * top // max(1, n - 1) if n > 1 else np.full(n, top)
        old = np.concatenate([np.zeros(p, np.int64), single]).astype(np.int64)
    return old, new


def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 16 + what)
    return g


def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(v).astype(np.int32)).cuda()


def _cache(case, seed, lens, held):
    """Pages with room for `lens` entries a sequence, of which `held` are there."""
    hq, hkv, d = HEADS[case["shard"]]
    ps, fmt = case["page"], case["fmt"]
    rng = np.random.default_rng([int(seed), 3])
    need = -(-lens // ps)
    width = max(1, int(need.max()))
    n_pages = int(need.sum()) + 1
    order = 1 + rng.permutation(n_pages - 1)
    table = np.zeros((len(lens), width), np.int32)
    named = np.arange(width)[None, :] < need[:, None]
    table[named] = order
    filled = np.zeros(n_pages, np.int64)
    filled[order] = np.clip(held[:, None] - ps * np.arange(width)[None, :], 0, ps)[named]
    s = {"op": case["op"], "hq": hq, "hkv": hkv, "d": d, "ps": ps, "fmt": fmt, "ks": FP8_K if fmt == "fp8" else 1.0,
         "vs": FP8_V if fmt == "fp8" else 1.0, "scales": None, "table": torch.from_numpy(table).cuda()}
    pages, scales = [], []
    for what, scale in ((0, FP8_K), (1, FP8_V)):
        x = torch.randn((n_pages, hkv, ps, d), generator=_gen(seed, what), device="cuda")
        if fmt == "int8":
            there = torch.arange(ps, device="cuda")[None, :] < torch.from_numpy(filled).cuda()[:, None]
            x = torch.where(there[:, None, :, None], x, 0.0).view(n_pages, hkv, ps // BLOCK, BLOCK, d)
            x = x * torch.exp(0.3 * torch.randn(x.shape[:3], generator=_gen(seed, 8 + what), device="cuda"))[..., None, None]
            f = x.abs().amax((3, 4)).clamp(min=LEAST) * (1 / 127)
            x = torch.round(x / f[..., None, None]).clamp(-127, 127).view(n_pages, hkv, ps, d)
            scales.append(f)
        pages.append((x / scale).to(torch.float8_e4m3fn) if fmt == "fp8" else x.to(torch.int8 if fmt == "int8" else torch.bfloat16))
    s["K"], s["V"] = pages
    if scales:
        s["scales"] = torch.stack(scales, dim=3)                # [n_pages, hkv, blocks of a page, 2]
    return s


def _rotary(d):
    f = 500000.0 ** (-np.arange(0, d, 2) / d)
    a = np.arange(POSITIONS)[:, None] * f[None, :]
    return [torch.from_numpy(t.astype(np.float32)).cuda() for t in (np.cos(a), np.sin(a))]


def _rows_out(s, n):
    return [torch.empty((n, s["hkv"] * s["d"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]


def _inputs(case, seed):
    rng = np.random.default_rng([int(seed), 2])
    if case["op"] in ("attend", "read"):
        lens = rng.permutation(_lens(case))
        s = _cache(case, seed, lens, lens)
        if case["op"] == "read":
            s["seqs"] = _i32(np.repeat(np.arange(len(lens)), lens))
            s["index"] = _i32(np.concatenate([np.arange(n) for n in lens]))
            s["k_out"], s["v_out"] = _rows_out(s, int(lens.sum()))
            return s
        s["lens"] = _i32(lens)
        s["q"] = (2 * torch.randn((len(lens), s["hq"] * s["d"]), generator=_gen(seed, 4), device="cuda")).to(torch.bfloat16)
        s["starts"] = torch.clamp(s["lens"] - case["window"], min=0) if case["window"] else None
        s["sinks"] = case["sinks"]
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((len(lens), s["hq"]), device="cuda")
        return s
    old, new = _counts(case)
    order = rng.permutation(len(old))
    old, new = old[order], new[order]
    T, begin = int(new.sum()), np.concatenate([[0], np.cumsum(new)])
    hq, hkv, d = HEADS[case["shard"]]
    if case["op"] == "prompt":
        s = _cache(case, seed, old + new, old + new)
        s["lens"], s["q_starts"], s["most"] = _i32(old + new), _i32(begin), int(new.max())
        # (the query part of the qkv projection's rows)
        rows = (2 * torch.randn((T, (hq + 2 * hkv) * d), generator=_gen(seed, 4), device="cuda")).to(torch.bfloat16)
        s["q"] = rows[:, :hq * d]
        s["window"], s["sinks"] = case["window"], case["sinks"]
        s["out"] = torch.empty((T, hq * d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((T, hq), device="cuda")
        return s
    s = _cache(case, seed, old + new, old)
    index = np.concatenate([np.arange(o, o + m) for o, m in zip(old, new)])
    s["seqs"], s["index"], s["positions"], s["lens"] = _i32(np.repeat(np.arange(len(new)), new)), _i32(index), _i32(index), _i32(old)
    s["cos"], s["sin"] = _rotary(d)
    s["qkv"] = torch.randn((T, (hq + 2 * hkv) * d), generator=_gen(seed, 4), device="cuda").to(torch.bfloat16)
    s["q_out"] = torch.empty((T, hq * d), dtype=torch.bfloat16, device="cuda")
    s["interleaved"], s["q_norm"], s["k_norm"] = case["interleaved"], None, None
    if case["norm"]:
        s["q_norm"], s["k_norm"] = ((1 + 0.2 * torch.randn(d, generator=_gen(seed, 5 + i), device="cuda")).to(torch.bfloat16)
                                    for i in range(2))
    if case["op"] == "store":
        # the entries of every block that the call writes into
        first = old // BLOCK * BLOCK
        s["read_seqs"] = _i32(np.repeat(np.arange(len(new)), old + new - first))
        s["read_index"] = _i32(np.concatenate([np.arange(f, o + m) for f, o, m in zip(first, old, new)]))
        s["k_out"], s["v_out"] = _rows_out(s, len(s["read_seqs"]))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2510_23346_amd as bd
        fmt = {"bf16": bd.KV_BF16, "fp8": bd.KV_FP8_E4M3, "int8": bd.KV_INT8}[s["fmt"]]
        s["kv"] = bd.KVCache(s["hq"], s["hkv"], s["d"], s["K"].shape[0], s["ps"], s["table"].shape[0], fmt=fmt,
                             k_scale=s["ks"], v_scale=s["vs"], k=s["K"], v=s["V"], scales=s["scales"])
    return s


def run(s):
    if s["op"] == "attend":
        if own:
            s["kv"].attend(s["q"], s["table"], s["lens"], s["out"], starts=s["starts"], sinks=s["sinks"], lse=s["lse"])
        else:
            _plain_attend(s)
        return {k: s[k] for k in ("out", "lse")}
    if s["op"] == "prompt":
        if own:
            s["kv"].attend_prompt(s["q"], s["q_starts"], s["table"], s["lens"], s["out"], window=s["window"], sinks=s["sinks"],
                                  lse=s["lse"])
        else:
            _plain_prompt(s)
        return {k: s[k] for k in ("out", "lse")}
    if s["op"] == "read":
        if own:
            s["kv"].read(s["seqs"], s["index"], s["table"], s["k_out"], s["v_out"])
        else:
            _plain_read(s, s["seqs"], s["index"])
        return {k: s[k] for k in ("k_out", "v_out")}
    if own:
        s["kv"].append(s["qkv"], s["cos"], s["sin"], s["seqs"], s["index"], s["positions"], s["table"], s["lens"], s["q_out"],
                       interleaved=s["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
    else:
        _plain_append(s)
    if s["op"] == "append":
        return {k: s[k] for k in ("q_out", "K", "V", "lens")}
    if own:
        s["kv"].read(s["read_seqs"], s["read_index"], s["table"], s["k_out"], s["v_out"])
    else:
        _plain_read(s, s["read_seqs"], s["read_index"])
    return {k: s[k] for k in ("q_out", "k_out", "v_out", "scales", "lens")}


# ---------------------------------------------------------------- plain forms

def _bits(x):
    """Rows of an e4m3 tensor can only be indexed as bytes."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _sequences(s):
    """Keys and values of every row of the page table: [B, hkv, width, d], fp32."""
    table = s["table"].long()
    B, hkv, width, d = table.shape[0], s["hkv"], table.shape[1] * s["ps"], s["d"]
    got = []
    for i, (x, scale) in enumerate(((s["K"], s["ks"]), (s["V"], s["vs"]))):
        y = _bits(x)[table].view(x.dtype).float() * scale                          # [B, pages, hkv, page, d]
        if s["scales"] is not None:
            y = y * s["scales"][table][..., i].repeat_interleave(BLOCK, 3)[..., None]
        got.append(y.transpose(1, 2).reshape(B, hkv, width, d))
    return got


def _softmax(score):
    """Probabilities and log of the sum; rows that see nothing: 0 and -inf."""
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    return torch.where(total > 0, p / total, 0.0), top + torch.log(total)


def _plain_attend(s):
    hq, hkv, d = s["hq"], s["hkv"], s["d"]
    K, V = _sequences(s)
    B, at = K.shape[0], torch.arange(K.shape[2], device="cuda")[None, :]
    seen = at < s["lens"][:, None]
    if s["starts"] is not None:
        seen = seen & ((at >= s["starts"][:, None]) | (at < s["sinks"]))
    q = s["q"].float().view(B, hkv, hq // hkv, d)
    score = torch.matmul(q, K.transpose(2, 3).contiguous()) * (1 / math.sqrt(d))
    p, lse = _softmax(score.masked_fill(~seen[:, None, None, :], -math.inf))
    s["out"].copy_(torch.matmul(p, V).reshape(B, hq * d))
    s["lse"].copy_(lse.view(B, hq))


def _plain_prompt(s):
    hq, hkv, d, most = s["hq"], s["hkv"], s["d"], s["most"]
    G, T = hq // hkv, s["q"].shape[0]
    K, V = _sequences(s)
    B, width = K.shape[0], K.shape[2]
    begin, lens = s["q_starts"].long(), s["lens"].long()
    count = begin[1:] - begin[:-1]
    i = torch.arange(most, device="cuda")[None, :]
    row = torch.clamp(begin[:-1, None] + i, max=T - 1)                               # [B, most]
    own_at = torch.where(i < count[:, None], lens[:, None] - count[:, None] + i, -1)  # the token's own entry; -1: no token
    at = torch.arange(width, device="cuda")[None, None, :]
    seen = at <= own_at[..., None]
    if s["window"]:
        seen = seen & ((at > own_at[..., None] - s["window"]) | (at < s["sinks"]))
    q = s["q"].float().view(T, hkv, G, d)[row].permute(0, 2, 3, 1, 4).reshape(B, hkv, G * most, d)
    score = torch.matmul(q, K.transpose(2, 3).contiguous()).mul_(1 / math.sqrt(d)).view(B, hkv, G, most, width)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    p, lse = _softmax(score)
    o = torch.matmul(p.view(B, hkv, G * most, width), V).view(B, hkv, G, most, d).permute(0, 3, 1, 2, 4).reshape(B * most, hq * d)
    # every row of q is a token of one sequence: where it is among the padded ones
    b = torch.searchsorted(begin[1:].contiguous(), torch.arange(T, device="cuda"), right=True)
    of = b * most + torch.arange(T, device="cuda") - begin[b]
    s["out"].copy_(o[of])
    s["lse"].copy_(lse.view(B, hq, most).transpose(1, 2).reshape(B * most, hq)[of])


def _place(s, seqs, index):
    seqs, index = seqs.long(), index.long()
    return s["table"][seqs, index // s["ps"]].long(), index % s["ps"]


def _plain_read(s, seqs, index):
    page, slot = _place(s, seqs, index)
    f = s["scales"][page, :, slot // BLOCK]                                          # [n, hkv, 2]
    s["k_out"].copy_((s["K"][page, :, slot].float() * f[..., 0:1]).flatten(1))
    s["v_out"].copy_((s["V"][page, :, slot].float() * f[..., 1:2]).flatten(1))


def _normed(x, w):
    return x * (1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)) * w.float()


def _plain_append(s):
    hq, hkv, d = s["hq"], s["hkv"], s["d"]
    x = s["qkv"].float().view(-1, hq + 2 * hkv, d)
    at = s["positions"].long()
    c, sn = s["cos"][at][:, None, :], s["sin"][at][:, None, :]
    r = x[:, :hq + hkv]
    if s["q_norm"] is not None:
        r = torch.cat([_normed(r[:, :hq], s["q_norm"]), _normed(r[:, hq:], s["k_norm"])], dim=1)
    if s["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * sn, b * c + a * sn], dim=-1).flatten(2)
    else:
        a, b = r[..., :d // 2], r[..., d // 2:]
        r = torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)
    s["q_out"].copy_(r[:, :hq].reshape(-1, hq * d))
    page, slot = _place(s, s["seqs"], s["index"])
    k, v = r[:, hq:], x[:, hq + hkv:]
    if s["fmt"] == "int8":
        _plain_store(s, page, slot, k, v)
    elif s["fmt"] == "fp8":
        for pages, y, scale in ((s["K"], k, s["ks"]), (s["V"], v, s["vs"])):
            y = (y * float(np.float32(1) / np.float32(scale))).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
            _bits(pages)[page, :, slot] = _bits(y)
    else:
        s["K"][page, :, slot] = k.to(torch.bfloat16)
        s["V"][page, :, slot] = v.to(torch.bfloat16)
    s["lens"].scatter_reduce_(0, s["seqs"].long(), s["index"] + 1, "amax")


def _plain_store(s, page, slot, k, v):
    """A block's scale is that of its largest number so far; a call that brings
    the first of its entries begins it anew.  What was there is rounded again
    where the scale grows."""
    hkv, d = s["hkv"], s["d"]
    n_pages, per = s["K"].shape[0], s["ps"] // BLOCK
    block = slot // BLOCK
    at = page * per + block
    size = torch.stack([k.abs().amax(2), v.abs().amax(2)], dim=2)                    # [T, hkv, 2]
    top = torch.zeros((n_pages * per, hkv, 2), device="cuda").scatter_reduce_(0, at[:, None, None].expand_as(size), size, "amax")
    anew = torch.zeros(n_pages * per, dtype=torch.int32, device="cuda").scatter_reduce_(0, at, (slot % BLOCK == 0).int(), "amax")
    anew = anew[at][:, None, None] > 0
    before = s["scales"][page, :, block]
    f = top[at].clamp(min=LEAST) * (1 / 127)
    f = torch.where(anew, f, torch.maximum(before, f))
    ratio = torch.where(anew, 1.0, before / f)
    s["scales"][page, :, block] = f
    rows = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")[None, :]      # [T, 16]
    heads = torch.arange(hkv, device="cuda")[None, :, None]
    for i, (pages, y) in enumerate(((s["K"], k), (s["V"], v))):
        whole = (page[:, None, None], heads, rows[:, None, :])
        pages[whole] = torch.round(pages[whole].float() * ratio[..., i, None, None]).to(torch.int8)
        pages[page, :, slot] = torch.round(y * (1 / f[..., i:i + 1])).clamp(-127, 127).to(torch.int8)


# ---------------------------------------------------------------- what a pass needs

def _pairs(old, new, window, sinks):
    """Entries that `new` tokens behind `old` entries see, all together."""
    p = np.arange(old, old + new)
    return int((p + 1 if not window else np.minimum(p + 1, np.minimum(window, p + 1) + np.minimum(sinks, np.maximum(0, p + 1 - window)))).sum())


def work(case):
    """Each entry that is attended to, appended or read once."""
    hq, hkv, d = HEADS[case["shard"]]
    # keys and values of one entry, and their share of the scales
    row = 2 * hkv * d * (2 if case["fmt"] == "bf16" else 1) + (8 * hkv / BLOCK if case["fmt"] == "int8" else 0)
    if case["op"] == "attend":
        n = _lens(case)
        if case["window"]:
            n = np.minimum(n, case["window"] + np.minimum(case["sinks"], np.maximum(0, n - case["window"])))
        n = int(n.sum())
        return {"bytes": float(n * row + 4 * -(-n // case["page"]) + case["B"] * (4 * hq * d + 4 * hq + 4)),
                "flops": float(4 * n * hq * d)}
    if case["op"] == "read":
        n = int(_lens(case).sum())
        return {"bytes": float(n * (row + 4 * hkv * d + 8)), "flops": float(2 * n * hkv * d)}
    old, new = _counts(case)
    T = int(new.sum())
    if case["op"] == "prompt":
        seen = old + new
        if case["window"]:
            seen = np.minimum(seen, case["window"] + new - 1 + np.minimum(case["sinks"], np.maximum(0, old + 1 - case["window"])))
        pairs = sum(_pairs(o, m, case["window"], case["sinks"]) for o, m in zip(old, new))
        return {"bytes": float(seen.sum() * row + T * (4 * hq * d + 4 * hq)), "flops": float(4 * pairs * hq * d)}
    nbytes = T * ((2 * hq + 2 * hkv) * d * 2 + row + 12) + 4 * d * int(min(T, (old + new).max())) + 4 * d
    if case["op"] == "store":
        n = int((old % BLOCK + new).sum())
        nbytes += n * (row + 4 * hkv * d + 8)
    return {"bytes": float(nbytes), "flops": float((8 if case["norm"] else 3) * T * (hq + hkv) * d)}


# ---------------------------------------------------------------- in 64 bits

def _values(s, pages, which, at):
    """Entries `at` = (pages, places) of a cache: [n, hkv, d]."""
    y = _bits(pages)[at[0], :, at[1]].view(pages.dtype).double()
    if s["scales"] is not None:
        return y * s["scales"][at[0], :, at[1] // BLOCK, which].double()[..., None]
    return y * (s["ks"], s["vs"])[which]


def exact(case, seed):
    s = _inputs(case, seed)
    table = s["table"].cpu().numpy().astype(np.int64)
    hq, hkv, d, ps = s["hq"], s["hkv"], s["d"], s["ps"]
    G = hq // hkv
    if case["op"] == "read":
        b, j = s["seqs"].cpu().numpy(), s["index"].cpu().numpy()
        at = tuple(torch.from_numpy(x).cuda() for x in (table[b, j // ps], (j % ps).astype(np.int64)))
        return {"k_out": _values(s, s["K"], 0, at).flatten(1), "v_out": _values(s, s["V"], 1, at).flatten(1)}
    if case["op"] in ("attend", "prompt"):
        lens = s["lens"].cpu().numpy().astype(np.int64)
        begin = s["q_starts"].cpu().numpy() if case["op"] == "prompt" else np.arange(len(lens) + 1)
        q = s["q"].double().view(-1, hkv, G, d)
        out = torch.zeros_like(q)
        lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(int(x) for x in lens):
            if n == 0:
                continue
            j = np.arange(n)
            at = tuple(torch.from_numpy(x).cuda() for x in (table[b, j // ps], j % ps))
            k, v = (_values(s, s["K"], 0, at), _values(s, s["V"], 1, at))
            for r0 in range(int(begin[b]), int(begin[b + 1]), 1024):
                r1 = min(int(begin[b + 1]), r0 + 1024)
                own_at = n - int(begin[b + 1]) + np.arange(r0, r1)
                hide = j[None, :] > own_at[:, None]
                if case["window"]:
                    hide |= (j[None, :] <= own_at[:, None] - case["window"]) & (j[None, :] >= case["sinks"])
                hide = torch.from_numpy(hide).cuda()
                for h in range(hkv):
                    for g in range(G):
                        a = (q[r0:r1, h, g] @ k[:, h].t().contiguous()) / math.sqrt(d)
                        a = a.masked_fill(hide, -math.inf)
                        lse[r0:r1, h, g] = torch.logsumexp(a, 1)
                        out[r0:r1, h, g] = torch.softmax(a, 1) @ v[:, h]
        return {"out": out.reshape(-1, hq * d), "lse": lse.reshape(-1, hq)}
    x = s["qkv"].double().view(-1, hq + 2 * hkv, d)
    if case["norm"]:
        for part, w in ((slice(0, hq), s["q_norm"]), (slice(hq, hq + hkv), s["k_norm"])):
            y = x[:, part]
            x[:, part] = y / (y.square().sum(2, keepdim=True) / d + EPS).sqrt() * w.double()
    b, index = s["seqs"].cpu().numpy(), s["index"].cpu().numpy()
    z = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()][:, None, :]
    h = d // 2
    i0, i1 = (slice(0, d, 2), slice(1, d, 2)) if case["interleaved"] else (slice(0, h), slice(h, d))
    turned = torch.complex(x[:, :hq + hkv, i0].contiguous(), x[:, :hq + hkv, i1].contiguous()) * z
    x[:, :hq + hkv, i0], x[:, :hq + hkv, i1] = turned.real, turned.imag
    out = {"q_out": x[:, :hq].reshape(-1, hq * d), "lens": None}
    page, slot = table[b, index // ps], index % ps
    rows = (x[:, hq:hq + hkv], x[:, hq + hkv:])
    if case["op"] == "append":
        for name, y, scale in (("K", rows[0], s["ks"]), ("V", rows[1], s["vs"])):
            pages = s[name].double()
            pages[page, :, slot] = y / scale
            out[name] = pages
        return out
    # block by block, as a queue of runs: (page, block) -> tokens
    pages = [s["K"].double(), s["V"].double()]
    scales = s["scales"].double()
    blocks = {}
    for t, key in enumerate(zip(page.tolist(), (slot // BLOCK).tolist())):
        blocks.setdefault(key, []).append(t)
    keys = np.array(list(blocks))
    tokens = np.full((len(keys), BLOCK), -1)
    for i, ts in enumerate(blocks.values()):
        tokens[i, slot[ts] % BLOCK] = ts
    new = torch.from_numpy(tokens >= 0).cuda()
    pg, bl = torch.from_numpy(keys[:, 0]).cuda(), torch.from_numpy(keys[:, 1]).cuda()
    place = bl[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    for which in (0, 1):
        y = rows[which][torch.from_numpy(np.maximum(tokens, 0)).cuda()].transpose(1, 2)        # [blocks, hkv, 16, d]
        mine = new[:, None, :, None]
        least = torch.where(mine, y.abs(), 0.0).amax((2, 3)).clamp(min=LEAST) / 127
        was = scales[pg, :, bl, which]
        now = torch.where(new[:, 0][:, None], least, torch.maximum(was, least))
        there = pages[which][pg[:, None], :, place].transpose(1, 2)
        there = torch.where(now[..., None, None] > was[..., None, None], torch.round(there * (was / now)[..., None, None]), there)
        there = torch.where(new[:, 0][:, None, None, None], pages[which][pg[:, None], :, place].transpose(1, 2), there)
        pages[which][pg[:, None], :, place] = torch.where(mine, torch.round(y / now[..., None, None]), there).transpose(1, 2)
        scales[pg, :, bl, which] = now
    rb, rj = s["read_seqs"].cpu().numpy(), s["read_index"].cpu().numpy()
    rp, rs = table[rb, rj // ps], rj % ps
    for which, name in ((0, "k_out"), (1, "v_out")):
        out[name] = (pages[which][rp, :, rs] * scales[rp, :, rs // BLOCK, which][..., None]).flatten(1)
    out["scales"] = scales
    return out
