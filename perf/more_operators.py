"""The operators of serving over a paged cache, as measurable cases.

A speculative step on tensors writes its new rows' keys and values into a
paged cache (pages of a power of two of tokens; elements as they are, or in
blocks of 32 that share a power of two), attends from those rows to the
cache, and adjusts the logits before tokens are picked.  Four operators:

  write   new rows of every sequence into the cache, then the same rows read
          back: the values that the cache now holds
  read    whole sequences out of the cache
  attn    attention of every sequence's new rows over its pages: causal, or
          within a window and to the first tokens ("sinks")
  logits  penalties for repeated tokens, biases and a grammar's mask, and the
          token with the largest logit left

A case is a plain dict.  ``run`` makes the plain computation in elementary
float32 torch operations, or, where ``own`` is set, the library's calls.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 32                          # elements that share a scale
# largest element of a block type, its exponent, bits of its fraction, smallest normal exponent
GRIDS = {"e4m3": (448.0, 8, 3, -6), "e2m1": (6.0, 2, 1, 0)}


def listed():
    return [
        # a verify pass of 32 conversations (K = 8) appends its rows: the call's latency
        dict(name="write_verify", kind="write", seqs=32, rows_lo=9, rows_hi=9, past_lo=512, past_hi=1024, hk=8, hd=64, page=16,
             dtype="bf16", cache="e4m3"),
        # prompts of a batch enter the cache, four bits an element
        dict(name="write_prompts_e2m1", kind="write", seqs=16, rows_lo=500, rows_hi=4096, past_lo=0, past_hi=0, hk=8, hd=128, page=64,
             dtype="bf16", cache="e2m1"),
        # one short sequence comes back: the call's latency
        dict(name="read_short", kind="read", seqs=1, rows_lo=70, rows_hi=70, past_lo=0, past_hi=0, hk=1, hd=64, page=16,
             dtype="bf16", cache="bf16"),
        # shared prefixes leave the cache for a pass that wants them in rows
        dict(name="read_prefix_e4m3", kind="read", seqs=8, rows_lo=1000, rows_hi=16384, past_lo=0, past_hi=0, hk=8, hd=128, page=32,
             dtype="f16", cache="e4m3"),
        # a token of the tiny pair's draft: the call's latency
        dict(name="attn_tiny", kind="attn", seqs=1, rows_lo=1, rows_hi=1, past_lo=69, past_hi=69, hq=2, hk=1, hd=64, page=16,
             dtype="bf16", cache="bf16", window=0, sinks=0),
        # a layer of the 8B-shaped target verifying K = 8 candidates of 32 ragged conversations
        dict(name="attn_verify", kind="attn", seqs=32, rows_lo=9, rows_hi=9, past_lo=512, past_hi=1536, hq=32, hk=8, hd=128, page=16,
             dtype="bf16", cache="bf16", window=0, sinks=0),
        # one long conversation, verified
        dict(name="attn_verify_16k", kind="attn", seqs=1, rows_lo=9, rows_hi=9, past_lo=16384, past_hi=16384, hq=32, hk=8, hd=128,
             page=64, dtype="f16", cache="f16", window=0, sinks=0),
        # single tokens of long contexts kept in eight bits
        dict(name="attn_decode_e4m3", kind="attn", seqs=16, rows_lo=1, rows_hi=1, past_lo=8000, past_hi=32000, hq=32, hk=8, hd=128,
             page=32, dtype="bf16", cache="e4m3", window=0, sinks=0),
        # chunks of prompts over what the cache has of them
        dict(name="attn_chunk", kind="attn", seqs=2, rows_lo=2048, rows_hi=4096, past_lo=4096, past_hi=8192, hq=32, hk=8, hd=128,
             page=64, dtype="bf16", cache="bf16", window=0, sinks=0),
        # the 1B-shaped draft within a window, first tokens kept, a cache of four bits; pages before the window are gone
        dict(name="attn_window_e2m1", kind="attn", seqs=24, rows_lo=1, rows_hi=300, past_lo=3000, past_hi=16000, hq=32, hk=8, hd=64,
             page=16, dtype="bf16", cache="e2m1", window=1024, sinks=4),
        # the verify pass of one conversation over the other family's vocabulary, 16-bit logits: the call's latency
        dict(name="logits_one", kind="logits", seqs=1, per=9, vocab=152064, past_lo=700, past_hi=700, dtype="bf16"),
        # the verify pass of 32 conversations
        dict(name="logits_batch", kind="logits", seqs=32, per=9, vocab=128256, past_lo=512, past_hi=1536, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["write", "read", "attn", "attn", "attn", "logits"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = rng.choice([dtype, dtype, "e4m3", "e4m3", "e2m1"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "logits":
        vocab = rng.choice([1024, 32000, 50257, 99991, 128256, 152064])
        dtype = rng.choice(["bf16", "f16", "f32"])
        rows = _log_int(rng, 1, 36_900_000 // vocab // (1 if dtype == "f32" else 2))
        per = rng.choice([1, 5, 9, 9, 13])
        hi = _log_int(rng, 1, 8192)
        return dict(kind="logits", seqs=max(1, min(rows, 2000) // per), per=per, vocab=vocab, past_lo=rng.randint(0, hi), past_hi=hi, dtype=dtype)
    if kind in ("write", "read"):
        hk, hd = rng.choice([(1, 64), (2, 64), (8, 64), (8, 128), (4, 128)])
        total = _log_int(rng, 1, 48_000_000 // (hk * hd))
        seqs = min(_log_int(rng, 1, 64), total)
        hi = max(1, total // seqs)
        past = rng.choice([0, _log_int(rng, 1, 4096)]) if kind == "write" else 0
        return dict(kind=kind, seqs=seqs, rows_lo=rng.randint(1, hi), rows_hi=hi, past_lo=rng.randint(0, past), past_hi=past, hk=hk, hd=hd,
                    page=page, dtype=dtype, cache=cache)
    hq, hk, hd = rng.choice([(2, 1, 64), (14, 2, 64), (32, 8, 64), (8, 8, 64), (32, 8, 128), (28, 4, 128), (5, 5, 128), (64, 2, 128)])
    rows = rng.choice([1, 1, 5, 9, 9, 13, 33, _log_int(rng, 1, 2048)])
    past = _log_int(rng, 1, 32000)
    # scores and keys of the padded batch: at most those of the listed cases
    most = min(3.2e9 / (hq * rows * (past + rows)), 5.2e8 / (hk * hd * (past + rows)))
    seqs = max(1, min(_log_int(rng, 1, 64), int(most)))
    window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
    return dict(kind="attn", seqs=seqs, rows_lo=rng.choice([rows, max(1, rows // 3)]), rows_hi=rows, past_lo=rng.randint(0, past),
                past_hi=past, hq=hq, hk=hk, hd=hd, page=page, dtype=dtype, cache=cache, window=window,
                sinks=rng.choice([0, 1, 4, 128]) if window else 0)


# --------------------------------------------------------------------------
# the cases' sequences (part of the case: every seed is the same work)
# --------------------------------------------------------------------------

def _sequences(case):
    """New rows and tokens before them of each sequence."""
    rng = random.Random(case["seqs"] * 1000003 + case["past_lo"] * 1009 + case["past_hi"] * 31 + case.get("rows_hi", 0))
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["seqs"])] if "rows_lo" in case else [case["per"]] * case["seqs"]
    return np.array(rows), np.array([rng.randint(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])])


def _first_seen(case, past):
    """First position that a sequence's rows see within their window."""
    return np.maximum(past - case["window"] + 1, 0) if case.get("window") else np.zeros_like(past)


# --------------------------------------------------------------------------
# the cache's formats
# --------------------------------------------------------------------------

def _pow2(e):
    """2^e in float32, e from -126 to 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _encode(x, cache):
    """Float32 [..., n] in blocks of 32 -> (codes, scale bytes).  A block's scale is
    the smallest 2^e, e >= -126, that brings it within the type's range."""
    top, _, fraction, low = GRIDS[cache]
    b = x.unflatten(-1, (-1, BLOCK))
    big = b.abs().amax(-1)
    m, ex = torch.frexp(big / top)                       # big / top = m 2^ex, 0.5 <= m < 1
    e = torch.where(m == 0.5, ex - 1, ex).clamp(min=-126)
    e = torch.where(big == 0, -126, e)
    # big / top is rounded: the smallest e is found next to it
    e = torch.where((big <= top * _pow2((e - 1).clamp(min=-126))), (e - 1).clamp(min=-126), e)
    e = torch.where(big > top * _pow2(e), e + 1, e)
    y = b * _pow2(-e)[..., None]
    step = _pow2((torch.frexp(y)[1] - 1).clamp(min=low) - fraction)
    y = (torch.round(y / step) * step).flatten(-2)       # (half to even)
    if cache == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)
    a = y.abs()
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, 7.0)).to(torch.uint8) | (y < 0).to(torch.uint8) * 8
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _decode(codes, scales, cache):
    """Float32 values of what `_encode` gives."""
    if cache == "e4m3":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        nibbles = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
        a = (nibbles & 7).float()
        a = torch.where(a <= 4, a / 2, torch.where(a <= 6, a - 2, 6.0))
        v = torch.where(nibbles >= 8, -a, a)
    return (v.unflatten(-1, (-1, BLOCK)) * _pow2(scales.to(torch.int32) - 127)[..., None]).flatten(-2)


# --------------------------------------------------------------------------
# prepare
# --------------------------------------------------------------------------

def _cache(case, g, positions_live):
    """Pages in any order, spare ones among them; what no sequence wrote holds anything."""
    hk, hd, page, seqs = case["hk"], case["hd"], case["page"], case["seqs"]
    rows, past = _sequences(case)
    need = -(-(rows + past) // page)                     # pages of each sequence
    width = int(need.max()) + 2
    n_pages = int(need.sum()) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")
    table = torch.randint(-(1 << 31), (1 << 31) - 1, (seqs, width), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    first = _first_seen(case, past) // page
    sinks = -(-case.get("sinks", 0) // page)
    at = torch.arange(width, device="cuda")[None]
    t = lambda a: torch.from_numpy(np.asarray(a)).cuda()[:, None]  # noqa: E731
    mine = at < t(need)
    seen = mine & ((at >= t(first)) | (at < sinks))      # the others are gone: their entries hold anything
    entry = order[(t(np.cumsum(need) - need) + at).clamp(max=n_pages - 1)].to(torch.int32)
    table = torch.where(seen, entry, table)
    shape = (n_pages, hk, page)
    s = dict(table=table, n_pages=n_pages)
    if case["cache"] in GRIDS:
        for name in ("k", "v"):
            s[name + "_cache"] = torch.randint(0, 256, (*shape, hd if case["cache"] == "e4m3" else hd // 2), generator=g, device="cuda",
                                               dtype=torch.uint8)
            s[name + "_scale"] = torch.randint(0, 256, (*shape, hd // BLOCK), generator=g, device="cuda", dtype=torch.uint8)
    else:
        for name in ("k", "v"):
            s[name + "_cache"] = torch.full((*shape, hd), math.nan, device="cuda", dtype=DTYPES[case["dtype"]])
            s[name + "_scale"] = None
    if positions_live:                                   # what earlier steps wrote
        pages = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
        pages[table[seen].long()] = True
        live = pages.nonzero()[:, 0]
        for name in ("k", "v"):
            for some in live.split(1 << 12):
                x = torch.randn(len(some), *shape[1:], hd, generator=g, device="cuda")
                if case["cache"] in GRIDS:
                    s[name + "_cache"][some], s[name + "_scale"][some] = _encode(x, case["cache"])
                else:
                    s[name + "_cache"][some] = x.to(DTYPES[case["dtype"]])
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "logits":
        return _prepare_logits(case, g)
    rows, past = _sequences(case)
    dt, hk, hd = DTYPES[case["dtype"]], case["hk"], case["hd"]
    n = int(rows.sum())
    s = dict(case=case, rows=n, scale=hd ** -0.5, **_cache(case, g, case["kind"] != "write"))
    s["row_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)])).to(torch.int32).cuda()
    s["kv_len"] = torch.from_numpy(rows + past).to(torch.int32).cuda()
    s["longest"] = int(rows.max())
    if case["kind"] == "attn":
        # the queries of one projection; its keys and values are in the cache by now
        hq = case["hq"]
        qkv = torch.randn(n, (hq + 2 * hk) * hd, generator=g, device="cuda").to(dt)
        s["q"] = qkv[:, :hq * hd].unflatten(1, (hq, hd))
    elif case["kind"] == "write":
        # a few channels lead, as keys' do
        kv = torch.randn(n, 2 * hk * hd, generator=g, device="cuda") * (1 + 8 * (torch.rand(2 * hk * hd, generator=g, device="cuda") > 0.97))
        kv = kv.to(dt)
        s["k"], s["v"] = kv[:, :hk * hd].unflatten(1, (hk, hd)), kv[:, hk * hd:].unflatten(1, (hk, hd))
    if own:
        # the handles of a cache, and of a step's batch, which every layer's calls take
        from paper_2504_18583_amd import binding as B
        s["handle"] = B.KVCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        s["batch"] = B.KVBatch(s["table"], s["row_start"], s["kv_len"], max_seq_rows=s["longest"])
    return s


def _prepare_logits(case, g):
    seqs, per, vocab = case["seqs"], case["per"], case["vocab"]
    n = seqs * per
    _, past = _sequences(case)
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case=case, logits=(torch.randn(n, vocab, generator=g, device="cuda") * 3).to(DTYPES[case["dtype"]]))
    # prompts and what was generated, few words often; then the candidates
    width = int(past.max()) + per
    s["tokens"] = (rand(seqs, width) ** 4 * vocab).to(torch.int32).clamp(max=vocab - 1)
    s["row_seq"] = torch.arange(n, device="cuda", dtype=torch.int32) // per
    s["row_len"] = torch.from_numpy(np.repeat(past, per) + np.tile(np.arange(per), seqs)).to(torch.int32).cuda()
    s["prompt_len"] = torch.from_numpy(past // 2).to(torch.int32).cuda()
    s["repetition"] = 1 + 0.5 * rand(seqs)
    s["presence"], s["frequency"] = rand(seqs), 0.5 * rand(seqs)
    # some sequences have biases, each on a few ids
    count = np.where(np.arange(seqs) % 3 == 0, 20 + np.arange(seqs) % 50, 0)
    ids = torch.randint(0, vocab, (int(count.sum()),), generator=g, device="cuda", dtype=torch.int32)
    first = np.concatenate([[0], np.cumsum(count)])
    for a, b in zip(first[:-1], first[1:]):              # an id once in a list
        ids[a:b] = torch.randperm(min(vocab, 1 << 14), generator=g, device="cuda")[:b - a].to(torch.int32)
    s["bias_start"] = torch.from_numpy(first).to(torch.int32).cuda()
    s["bias_ids"], s["bias_values"] = ids, 4 * torch.randn(len(ids), generator=g, device="cuda")
    # a grammar leaves some tokens; every fourth sequence has none
    words = -(-vocab // 32)
    s["mask"] = torch.randint(-(1 << 31), (1 << 31) - 1, (n, words), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    at = torch.arange(n, device="cuda", dtype=torch.int32)
    s["mask_row"] = torch.where(s["row_seq"] % 4 == 3, -1, at).to(torch.int32)
    if n > 2:
        s["mask"][n // 2] = 0                            # a state that allows nothing
    s["out"] = torch.empty_like(s["logits"])
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------

def _places(s):
    """Sequence and position of every row."""
    start, at = s["row_start"].long(), torch.arange(s["rows"], device="cuda")
    seq = (at[:, None] >= start[None, 1:]).sum(1)
    return seq, s["kv_len"].long()[seq] - start[seq + 1] + at


def _slots(s, seq, pos):
    """Page and place in it of positions of sequences."""
    page = s["case"]["page"]
    return s["table"].long()[seq, pos // page], pos % page


def _write_plain(s):
    page, place = _slots(s, *_places(s))
    for name in ("k", "v"):
        if s["case"]["cache"] in GRIDS:
            s[name + "_cache"][page, :, place], s[name + "_scale"][page, :, place] = _encode(s[name].float(), s["case"]["cache"])
        else:
            s[name + "_cache"][page, :, place] = s[name]


def _values(s, name, page, place):
    """Float32 values at places of the cache."""
    x = s[name + "_cache"][page, :, place]
    if s["case"]["cache"] in GRIDS:
        return _decode(x, s[name + "_scale"][page, :, place], s["case"]["cache"])
    return x.float()


def _read_plain(s):
    page, place = _slots(s, *_places(s))
    return {name: _values(s, name, page, place).to(DTYPES[s["case"]["dtype"]]) for name in ("k", "v")}


def _attn_plain(s):
    case = s["case"]
    hk, hd, window, sinks = case["hk"], case["hd"], case["window"], case["sinks"]
    start, end = s["row_start"].long()[:-1], s["row_start"].long()[1:]
    rows, kv_len = end - start, s["kv_len"].long()
    n, m, length = case["seqs"], s["longest"], s["table"].shape[1] * case["page"]
    i, j = torch.arange(m, device="cuda"), torch.arange(length, device="cuda")
    valid = i[None] < rows[:, None]
    idx = torch.where(valid, start[:, None] + i[None], 0)
    pos = (kv_len - rows)[:, None] + i[None]             # [sequences, rows]
    seen = j[None, None] <= pos[..., None]
    if window:
        seen = seen & ((j[None, None] > pos[..., None] - window) | (j < sinks)[None, None])
    seen = seen & valid[..., None]
    used = seen.any(1)                                   # [sequences, keys]
    page, place = _slots(s, torch.arange(n, device="cuda")[:, None], j[None].expand(n, -1))
    page = torch.where(used, page, 0)
    k = _values(s, "k", page, place).masked_fill_(~used[..., None, None], 0.0).permute(0, 2, 3, 1).contiguous()
    q = s["q"].float()[idx].permute(0, 2, 1, 3).reshape(n, hk, -1, hd)
    p = torch.matmul(q, k).view(n, hk, -1, m, length).mul_(s["scale"])
    del k
    p.masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    norm = p.sum(-1, keepdim=True)
    p.div_(torch.where(norm == 0, 1.0, norm))
    v = _values(s, "v", page, place).masked_fill_(~used[..., None, None], 0.0).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.view(n, hk, -1, length), v).view(n, -1, m, hd)
    lse = (top + torch.log(norm)).view(n, -1, m)
    out = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    out[idx[valid]] = o.permute(0, 2, 1, 3)[valid].to(out.dtype)
    by_row = torch.empty(case["hq"], s["rows"], device="cuda")
    by_row[:, idx[valid]] = lse.permute(1, 0, 2)[:, valid]
    return {"out": out, "lse": by_row}


def _logits_plain(s):
    case = s["case"]
    vocab, seq = case["vocab"], s["row_seq"].long()
    x = s["logits"].float()
    n = len(x)
    tokens = s["tokens"].long()[seq]                     # [rows, history]
    at = torch.arange(tokens.shape[1], device="cuda")[None]
    there = at < s["row_len"][:, None]
    count = torch.zeros(n, vocab, device="cuda")
    count.scatter_add_(1, tokens, (there & (at >= s["prompt_len"].long()[seq][:, None])).float())
    known = torch.zeros(n, vocab, device="cuda").scatter_add_(1, tokens, there.float()) > 0
    r = s["repetition"][seq][:, None]
    x = torch.where(known, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][seq][:, None] * count
    x = x - s["presence"][seq][:, None] * (count > 0)
    lists = (torch.arange(len(s["bias_ids"]), device="cuda")[:, None] >= s["bias_start"].long()[None, 1:]).sum(1)
    bias = torch.zeros(case["seqs"], vocab, device="cuda")
    bias[lists, s["bias_ids"].long()] = s["bias_values"]
    x = x + bias[seq]
    words = s["mask"].long()[s["mask_row"].long().clamp(min=0)]
    allowed = ((words[..., None] >> torch.arange(32, device="cuda")) & 1).flatten(1)[:, :vocab] == 1
    x = x.masked_fill(~allowed & (s["mask_row"] >= 0)[:, None], -math.inf)
    s["out"].copy_(x)
    y = s["out"].float()
    top = y.amax(-1, keepdim=True)
    first = torch.where(y == top, torch.arange(vocab, device="cuda"), vocab).amin(-1)
    return {"logits": s["out"], "best": torch.where(torch.isinf(top[:, 0]), -1, first).to(torch.int32)}


# --------------------------------------------------------------------------
# run
# --------------------------------------------------------------------------

def _run_own(s):
    from paper_2504_18583_amd import binding as B
    case = s["case"]
    if case["kind"] == "attn":
        out, lse = B.kv_attn(s["q"], s["handle"], s["batch"], s["scale"], window=case["window"], sinks=case["sinks"])
        return {"out": out, "lse": lse}
    if case["kind"] == "logits":
        out, best = B.logits_adjust(s["logits"], s["tokens"], s["row_len"], s["prompt_len"], row_seq=s["row_seq"],
                                    repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"],
                                    bias=(s["bias_start"], s["bias_ids"], s["bias_values"]), mask=s["mask"], mask_row=s["mask_row"],
                                    out=s["out"])
        return {"logits": out, "best": best}
    if case["kind"] == "write":
        B.kv_write(s["k"], s["v"], s["handle"], s["batch"])
    k, v = B.kv_read(s["handle"], s["batch"], s["rows"], DTYPES[case["dtype"]])
    return {"k": k, "v": v}


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "attn":
        return _attn_plain(s)
    if kind == "logits":
        return _logits_plain(s)
    if kind == "write":
        _write_plain(s)
    return _read_plain(s)


# --------------------------------------------------------------------------
# work
# --------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    rows, past = _sequences(case)
    n = float(rows.sum())
    if case["kind"] == "logits":
        masked = sum(1 for i in range(case["seqs"]) if i % 4 != 3) * case["per"]
        n_bytes = 2.0 * n * case["vocab"] * size + masked * case["vocab"] / 8 + 4.0 * (past.sum() + 2 * n)
        return {"bytes": float(n_bytes), "flops": 8.0 * n * case["vocab"]}
    hk, hd = case["hk"], case["hd"]
    held = {"e4m3": 1 + 1 / BLOCK, "e2m1": 0.5 + 1 / BLOCK}.get(case["cache"], 2.0)     # bytes of a cached element
    if case["kind"] != "attn":
        passes = 2 if case["kind"] == "write" else 1
        return {"bytes": passes * 2.0 * n * hk * hd * (size + held), "flops": passes * 8.0 * n * hk * hd}
    hq, window, sinks = case["hq"], case["window"], case["sinks"]
    pairs = keys = 0.0
    for m, p in zip(rows, past):
        pos = p + np.arange(m, dtype=np.float64)
        if window:
            pairs += (np.minimum(pos + 1, window) + np.clip(pos + 1 - window, 0, sinks)).sum()
            first = max(p - window + 1, 0)
            keys += p + m - first + min(sinks, first)
        else:
            pairs += (pos + 1).sum()
            keys += p + m
    return {"bytes": float(keys * 2.0 * hk * hd * held + n * hq * (2.0 * hd * size + 4)), "flops": float(4.0 * pairs * hd * hq)}


# --------------------------------------------------------------------------
# exact: the definitions in float64
# --------------------------------------------------------------------------

def _grid(cache):
    """The magnitudes that a code's low bits stand for, ascending."""
    _, _, fraction, low = GRIDS[cache]
    codes = range(127 if cache == "e4m3" else 8)
    ones = 1 << fraction
    return torch.tensor([(c % ones) / ones * 2.0 ** low if c < ones else (1 + (c % ones) / ones) * 2.0 ** (c // ones - 1 + low) for c in codes],
                        dtype=torch.float64, device="cuda")


def _stored_exact(x, cache):
    """What blocks of 32 are stored as: the nearest grid value under the block's scale, to an even code at halves."""
    grid = _grid(cache)
    b = x.double().unflatten(-1, (-1, BLOCK))
    scale = torch.full_like(b[..., :1], 2.0 ** -126)
    big = b.abs().amax(-1, keepdim=True)
    for _ in range(254):                                 # the smallest power of two that holds the block
        short = big > grid[-1] * scale
        if not bool(short.any()):
            break
        scale = torch.where(short, scale * 2, scale)
    a = (b / scale).abs()
    above = torch.searchsorted(grid, a.contiguous()).clamp(max=len(grid) - 1)
    below = (above - 1).clamp(min=0)
    up, down = grid[above] - a, a - grid[below]
    pick = torch.where(up < down, above, torch.where(down < up, below, torch.where(above % 2 == 0, above, below)))
    return (torch.copysign(grid[pick], b) * scale).flatten(-2)


def _held_exact(s, name, page, place):
    """Float64 values at places of the cache, by a table of the codes."""
    cache, x = s["case"]["cache"], s[name + "_cache"][page, :, place]
    if cache not in GRIDS:
        return x.double()
    grid = _grid(cache)
    if cache == "e4m3":
        table = torch.cat([grid, torch.tensor([math.nan], dtype=torch.float64, device="cuda")])
        v = torch.cat([table, -table])[x.long()]
    else:
        v = torch.cat([grid, -grid])[torch.stack([x % 16, x // 16], -1).flatten(-2).long()]
    scale = torch.exp2(s[name + "_scale"][page, :, place].double() - 127)
    return v * scale.repeat_interleave(BLOCK, -1)


def _rows_exact(s):
    rows, past = _sequences(s["case"])
    seq = torch.from_numpy(np.repeat(np.arange(len(rows)), rows)).cuda()
    pos = torch.from_numpy(np.concatenate([p + np.arange(m) for m, p in zip(rows, past)])).cuda()
    return _slots(s, seq, pos)


def _attn_exact(s):
    case = s["case"]
    hq, group, window, sinks = case["hq"], case["hq"] // case["hk"], case["window"], case["sinks"]
    out = torch.zeros(s["rows"], hq, case["hd"], device="cuda", dtype=torch.float64)
    lse = torch.zeros(hq, s["rows"], device="cuda", dtype=torch.float64)
    at = 0
    for i, (m, p) in enumerate(zip(*_sequences(case))):
        pos = int(p) + torch.arange(int(m), device="cuda")[:, None]
        key = torch.arange(int(p + m), device="cuda")
        if window:
            key = key[(key >= int(p) - window + 1) | (key < sinks)]
        hidden = key[None] > pos
        if window:
            hidden |= (key[None] <= pos - window) & (key[None] >= sinks)
        page, place = _slots(s, torch.full_like(key, i), key)
        k, v = _held_exact(s, "k", page, place), _held_exact(s, "v", page, place)
        rows = slice(at, at + int(m))
        for h in range(hq):
            sc = torch.matmul(s["q"][rows, h].double(), k[:, h // group].T.contiguous()).mul_(s["scale"]).masked_fill_(hidden, -math.inf)
            lse[h, rows] = torch.logsumexp(sc, -1)
            out[rows, h] = torch.matmul(torch.softmax(sc, -1), v[:, h // group].contiguous())
        at += int(m)
    return {"out": out, "lse": lse}


def _logits_exact(s):
    case = s["case"]
    n, vocab = s["logits"].shape
    y = s["logits"].double()
    seqs = s["row_seq"].tolist()
    for r, (q, length, mask) in enumerate(zip(seqs, s["row_len"].tolist(), s["mask_row"].tolist())):
        history = s["tokens"][q, :length].long()
        made = torch.bincount(history[int(s["prompt_len"][q]):], minlength=vocab).double()
        old = torch.unique(history)
        rep = s["repetition"][q].double()
        y[r, old] = torch.where(y[r, old] > 0, y[r, old] / rep, y[r, old] * rep)
        y[r] -= s["frequency"][q].double() * made + s["presence"][q].double() * made.sign()
        a, b = int(s["bias_start"][q]), int(s["bias_start"][q + 1])
        y[r].index_add_(0, s["bias_ids"][a:b].long(), s["bias_values"][a:b].double())
        if mask >= 0:
            bits = s["mask"][mask].long() & 0xffffffff
            token = torch.arange(vocab, device="cuda")
            y[r][torch.div(bits[token // 32], 2 ** (token % 32), rounding_mode="floor") % 2 == 0] = -math.inf
    return {"logits": y, "best": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "logits":
        return _logits_exact(s)
    if case["kind"] == "attn":
        return _attn_exact(s)
    if case["kind"] == "read":
        page, place = _rows_exact(s)
        return {name: _held_exact(s, name, page, place) for name in ("k", "v")}
    if case["cache"] in GRIDS:
        return {name: _stored_exact(s[name], case["cache"]) for name in ("k", "v")}
    return {name: s[name].double() for name in ("k", "v")}
