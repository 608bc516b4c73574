"""The operators of mask-token training, as measurable cases.

A draft is trained on the packed rows that ``pard_cod_build`` writes: row
(k, j) is column j of subtask k of its sample (k = 1: a real token, k >= 2: a
mask token), at position j.  Three operators stand between the projections of
such a training step:

  rope   rotary positions of queries and keys (optionally normalised per head
         in the same pass), forward or gradient
  attn   attention over the packed rows: real tokens up to the row's context
         and the masks before it on its diagonal; forward, or forward and
         gradient ("train")
  loss   the mask-token loss (mean over each subtask's rows) and its gradient

A case is a plain dict.  ``run`` makes the plain computation in elementary
float32 torch operations, or, where ``own`` is set, the library's calls.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

RETAIN, RETAIN_MIN = 0.7, 0.2      # COD retention (the library's benchmark setting)
# rotary scalings: factor, low and high (bounds in turns of the original context), original context
SCALINGS = {"linear": (2.0,), "llama3": (8.0, 1.0, 4.0, 8192), "yarn": (4.0, 1.0, 32.0, 4096)}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # the tiny draft's rows of one short sample: the call's latency
        dict(name="rope_tiny", kind="rope", rows=67, hq=2, hk=1, hd=64, rot=64, layout="half", scaling="none",
             theta=1e4, dtype="bf16", norm=False, grad=False, max_pos=64),
        # a layer of the 1B-shaped draft over a batch of 16 packed samples
        dict(name="rope_1b", kind="rope", rows=34500, hq=32, hk=8, hd=64, rot=64, layout="half",
             scaling="llama3", theta=5e5, dtype="bf16", norm=False, grad=False, max_pos=1024),
        # the backward pass of 8B-shaped heads with per-head norms
        dict(name="rope_norm_grad", kind="rope", rows=8191, hq=32, hk=8, hd=128, rot=128, layout="half",
             scaling="none", theta=1e6, dtype="bf16", norm=True, grad=True, max_pos=8192),
        # interleaved pairs over part of the head, far positions, float32
        dict(name="rope_part_f32", kind="rope", rows=5003, hq=14, hk=2, hd=64, rot=32, layout="interleaved",
             scaling="yarn", theta=1e4, dtype="f32", norm=True, grad=False, max_pos=131072),
        # two short samples through the tiny draft's heads: the call's latency
        dict(name="attn_tiny", kind="attn", samples=2, lo=17, hi=40, k=4, hq=2, hk=1, hd=64, dtype="bf16",
             train=False),
        # a layer of the 1B-shaped draft, the paper's batch and lengths (512 to 1024 tokens, K = 8)
        dict(name="attn_1b", kind="attn", samples=16, lo=256, hi=1024, k=8, hq=32, hk=8, hd=64, dtype="bf16",
             train=False),
        # the same with its backward pass
        dict(name="attn_1b_train", kind="attn", samples=16, lo=256, hi=1024, k=8, hq=32, hk=8, hd=64,
             dtype="bf16", train=True),
        # 8B-shaped heads (head_dim 128), ragged documents, forward and backward
        dict(name="attn_8b_train", kind="attn", samples=6, lo=900, hi=2048, k=8, hq=32, hk=8, hd=128,
             dtype="f16", train=True),
        # the longest sample the data processing makes
        dict(name="attn_8k", kind="attn", samples=1, lo=8193, hi=8193, k=8, hq=8, hk=4, hd=64, dtype="bf16",
             train=False),
        # the tiny pair's vocabulary, float32 logits: the call's latency
        dict(name="loss_tiny", kind="loss", rows=134, vocab=1024, k=4, dtype="f32", grad=True, scale=1.0),
        # the draft's loss over its full vocabulary, with the gradient
        dict(name="loss_1b", kind="loss", rows=4099, vocab=128256, k=8, dtype="bf16", grad=True, scale=1.0),
        # evaluation over the other family's vocabulary, no gradient
        dict(name="loss_eval_qwen", kind="loss", rows=2050, vocab=152064, k=8, dtype="f16", grad=False, scale=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["rope", "attn", "attn", "loss"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "rope":
        hq, hk, hd = rng.choice([(2, 1, 64), (32, 8, 64), (14, 2, 64), (32, 8, 128), (28, 4, 128), (12, 12, 96),
                                 (5, 1, 80), (8, 4, 256)])
        dtype = rng.choice(["bf16", "f16", "f32"])
        rows = _log_int(rng, 1, 80_000_000 // ((hq + hk) * hd) // (2 if dtype == "f32" else 1))
        return dict(kind="rope", rows=rows, hq=hq, hk=hk, hd=hd, rot=rng.choice([hd, hd, hd // 2]),
                    layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "llama3", "yarn"]), theta=rng.choice([1e4, 5e5, 1e6]),
                    dtype=dtype, norm=rng.random() < 0.5, grad=rng.random() < 0.5, max_pos=_log_int(rng, 64, 131072))
    if kind == "attn":
        hq, hk, hd = rng.choice([(2, 1, 64), (4, 2, 64), (32, 8, 64), (14, 2, 64), (8, 8, 64), (32, 8, 128),
                                 (28, 4, 128), (4, 1, 128)])
        k = rng.choice([1, 2, 4, 8, 8, 12])
        hi = _log_int(rng, 2, 2048)
        # scores of the padded batch: at most those of the listed cases
        cap = _rows_cap(hi, k)
        most = int(4.5e9 / (hq * cap * cap))
        samples = min(_log_int(rng, 1, 48), max(1, most))
        return dict(kind="attn", samples=samples, lo=rng.randint(2, hi), hi=hi, k=k, hq=hq, hk=hk, hd=hd, dtype=dtype,
                    train=rng.random() < 0.5)
    vocab = rng.choice([1024, 4096, 32000, 50257, 128256, 152064, 99991])
    dtype = rng.choice(["bf16", "f16", "f32"])
    rows = _log_int(rng, 1, 500_000_000 // vocab // (2 if dtype == "f32" else 1))
    return dict(kind="loss", rows=min(rows, 60000), vocab=vocab, k=rng.choice([1, 4, 8, 12]), dtype=dtype,
                grad=rng.random() < 0.7, scale=1024.0 if dtype == "f16" else 1.0)


# --------------------------------------------------------------------------
# packed rows
# --------------------------------------------------------------------------

def _keep_counts(n, k):
    out, gamma = [n], 1.0
    for _ in range(2, k + 1):
        gamma *= RETAIN
        out.append(int(math.floor(n * max(gamma, RETAIN_MIN) + 0.5)))
    return out


def _rows_cap(n_tokens, k):
    """Packed rows that a sample of n_tokens tokens may need."""
    return sum(_keep_counts(n_tokens - 1, k))


def _lengths(case):
    """Tokens of each sample (part of the case: every seed is the same work)."""
    rng = random.Random(case["samples"] * 1000003 + case["lo"] * 1009 + case["hi"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["samples"])]


def _offsets(case):
    return np.concatenate([[0], np.cumsum([_rows_cap(n, case["k"]) for n in _lengths(case)])]).astype(np.int64)


def _pack(case, seed):
    """(section, column, length) of the packed rows: subtask k >= 2 keeps a random
    part of the columns whose predecessor subtask k - 1 kept."""
    rng = np.random.default_rng(seed)
    offs = _offsets(case)
    section, column = np.zeros(offs[-1], np.int32), np.zeros(offs[-1], np.int32)
    lens = np.zeros(len(offs) - 1, np.int32)
    for s, tokens in enumerate(_lengths(case)):
        n, at = tokens - 1, int(offs[s])
        kept = np.arange(n)
        for k, target in enumerate(_keep_counts(n, case["k"]), start=1):
            if k > 1:
                valid = kept[kept < n - 1] + 1
                kept = np.sort(rng.permutation(valid)[:target])
            section[at:at + len(kept)] = k
            column[at:at + len(kept)] = kept
            at += len(kept)
        lens[s] = at - offs[s]
    return section, column, lens


# --------------------------------------------------------------------------
# prepare
# --------------------------------------------------------------------------

def _inverse_frequencies(case):
    """Rotary frequencies in float64, and the factor on cosines and sines."""
    rot, theta, sc = case["rot"], case["theta"], case["scaling"]
    i = np.arange(rot // 2, dtype=np.float64)
    w = theta ** (-2.0 * i / rot)
    if sc == "none":
        return w, 1.0
    if sc == "linear":
        return w / SCALINGS[sc][0], 1.0
    factor, low, high, orig = SCALINGS[sc]
    if sc == "llama3":
        turns = orig * w / (2 * math.pi)
        s = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return (1 - s) * w / factor + s * w, 1.0
    # YaRN: full extrapolation above `high` turns of the original context, full
    # interpolation below `low`, a ramp over the dimensions between
    dim = lambda turns: rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    first, last = max(math.floor(dim(high)), 0), min(math.ceil(dim(low)), rot - 1)
    ramp = np.clip((i - first) / max(last - first, 1e-3), 0.0, 1.0)
    return w / factor * ramp + w * (1 - ramp), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    randn = lambda *shape, std=1.0, dtype=dt: (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    if case["kind"] == "rope":
        rows, hq, hk, hd = case["rows"], case["hq"], case["hk"], case["hd"]
        # queries, keys and values as one projection leaves them
        qkv = randn(rows, (hq + 2 * hk) * hd)
        s = dict(case=case, q=qkv[:, :hq * hd].unflatten(1, (hq, hd)),
                 k=qkv[:, hq * hd:(hq + hk) * hd].unflatten(1, (hk, hd)))
        s["pos"] = torch.randint(0, case["max_pos"], (rows,), generator=g, device="cuda", dtype=torch.int32)
        w, m = _inverse_frequencies(case)
        a = torch.arange(case["max_pos"], device="cuda", dtype=torch.float64)[:, None] * torch.from_numpy(w).cuda()
        s["table"] = torch.stack([torch.cos(a) * m, torch.sin(a) * m], -1).float()
        s["gq"] = 1 + randn(hd, std=0.1, dtype=torch.float32) if case["norm"] else None
        s["gk"] = 1 + randn(hd, std=0.1, dtype=torch.float32) if case["norm"] else None
        s["eps"] = 1e-6
        if case["grad"]:
            s["dq"], s["dk"] = randn(rows, hq, hd), randn(rows, hk, hd)
        return s
    if case["kind"] == "loss":
        rows, vocab = case["rows"], case["vocab"]
        logits = randn(rows, vocab, std=2.0)
        labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        # a model in training: the label's logit leads in some rows; every 61st row is padding
        logits[torch.arange(rows, device="cuda"), labels] += randn(rows, std=4.0).abs()
        section = torch.randint(1, case["k"] + 1, (rows,), generator=g, device="cuda").to(torch.int32)
        labels = torch.where(torch.arange(rows, device="cuda") % 61 == 60, -1, labels).to(torch.int32)
        return dict(case=case, logits=logits, labels=labels, section=section,
                    weights=[1.0 / case["k"]] * case["k"], d_logits=torch.empty_like(logits) if case["grad"] else None)
    section, column, lens = _pack(case, seed)
    rows, hq, hk, hd = len(section), case["hq"], case["hk"], case["hd"]
    qkv = randn(rows, (hq + 2 * hk) * hd)
    s = dict(case=case, q=qkv[:, :hq * hd].unflatten(1, (hq, hd)), k=qkv[:, hq * hd:(hq + hk) * hd].unflatten(1, (hk, hd)),
             v=qkv[:, (hq + hk) * hd:].unflatten(1, (hk, hd)), scale=hd ** -0.5, offsets=_offsets(case),
             section=torch.from_numpy(section).cuda(), column=torch.from_numpy(column).cuda(),
             lens=torch.from_numpy(lens).cuda())
    if case["train"]:
        s["d_out"] = randn(rows, hq, hd)
    if own:
        # built once for a batch, then used by every layer's forward and backward call
        from paper_2504_18583_amd import binding as B
        s["plan"] = B.cod_plan(s["section"], s["column"], s["offsets"], s["lens"])
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------

def _rotated(x, cos, sin, layout):
    """Rotation of the first 2 * cos.shape[-1] dims of x [rows, heads, hd]."""
    half = cos.shape[-1]
    if layout == "half":
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _rope_plain(x, gain, s):
    cs = s["table"][s["pos"].long()][:, None]
    x32 = x.float()
    if gain is not None:
        x32 = x32 * torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + s["eps"]) * gain
    return _rotated(x32, cs[..., 0], cs[..., 1], s["case"]["layout"]).to(x.dtype)


def _rope_grad_plain(dy, x, gain, s):
    cs = s["table"][s["pos"].long()][:, None]
    dn = _rotated(dy.float(), cs[..., 0], -cs[..., 1], s["case"]["layout"])
    if gain is None:
        return dn.to(x.dtype), None
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + s["eps"])
    xh = x32 * r
    dg = (dn * xh).sum((0, 1), dtype=torch.float64).float()
    t = dn * gain
    return (r * (t - xh * (t * xh).mean(-1, keepdim=True))).to(x.dtype), dg


def _padded(s):
    """Row index [samples, longest] of the packed batch and which entries are rows."""
    offs = torch.from_numpy(s["offsets"]).cuda()
    i = torch.arange(int(np.diff(s["offsets"]).max()), device="cuda")
    valid = i[None] < s["lens"][:, None]
    return torch.where(valid, offs[:-1, None] + i[None], 0), valid


def _scores(s, idx, valid):
    """Masked float32 scores [samples, key heads, group, rows, rows]."""
    hk, hd = s["k"].shape[1:]
    n, m = idx.shape
    sec, d = s["section"][idx], (s["column"] - s["section"])[idx]
    trunk = (sec == 1)[:, None, :] & (d[:, None, :] <= d[:, :, None])
    chain = (d[:, None, :] == d[:, :, None]) & (sec[:, None, :] <= sec[:, :, None])
    seen = (trunk | ((sec > 1)[:, None, :] & chain)) & valid[:, None, :] & valid[:, :, None]
    q = s["q"].float()[idx].permute(0, 2, 1, 3).reshape(n, hk, -1, hd)        # head-major within the group
    k = s["k"].float()[idx].permute(0, 2, 3, 1).contiguous()
    sc = torch.matmul(q, k).view(n, hk, -1, m, m).mul_(s["scale"])
    return sc.masked_fill_(~seen[:, None, None], -math.inf)


def _rows_back(x, like, idx, valid):
    """[samples, heads, longest, hd] -> packed rows, zeros where no row is."""
    out = torch.zeros(like.shape[0], x.shape[1], x.shape[3], device="cuda", dtype=torch.float32)
    out[idx[valid]] = x.permute(0, 2, 1, 3)[valid]
    return out.to(like.dtype)


def _attn_plain(s):
    idx, valid = _padded(s)
    n, m = idx.shape
    rows, hq, hd = s["q"].shape
    hk = s["k"].shape[1]
    p = _scores(s, idx, valid)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    norm = p.sum(-1, keepdim=True)
    p.div_(torch.where(norm == 0, 1.0, norm))
    v = s["v"].float()[idx].permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.view(n, hk, -1, m), v).view(n, hq, m, hd)
    lse = torch.full((hq, rows), -math.inf, device="cuda")
    lse[:, idx[valid]] = (top + torch.log(norm)).view(n, hq, m).permute(1, 0, 2)[:, valid]
    res = {"out": _rows_back(o, s["q"], idx, valid), "lse": lse}
    if not s["case"]["train"]:
        return res
    do = s["d_out"].float()[idx].permute(0, 2, 1, 3).reshape(n, hk, -1, hd)
    do = do * valid[:, None, :].expand(n, hq // hk, m).reshape(n, 1, -1, 1)
    dv = torch.matmul(p.view(n, hk, -1, m).transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_((do * o.view(n, hk, -1, hd)).sum(-1, keepdim=True))
    ds.mul_(p.view(n, hk, -1, m)).mul_(s["scale"])
    del p
    k = s["k"].float()[idx].permute(0, 2, 1, 3).contiguous()
    q = s["q"].float()[idx].permute(0, 2, 1, 3).reshape(n, hk, -1, hd)
    dq = torch.matmul(ds, k).view(n, hq, m, hd)
    dk = torch.matmul(ds.transpose(2, 3), q)
    return res | {"dq": _rows_back(dq, s["q"], idx, valid), "dk": _rows_back(dk, s["k"], idx, valid),
                  "dv": _rows_back(dv, s["v"], idx, valid)}


def _loss_plain(s):
    case = s["case"]
    x = s["logits"].float()
    labels, section = s["labels"].long(), s["section"].long()
    counted = labels >= 0
    top = x.amax(-1, keepdim=True)
    e = (x - top).exp_()
    norm = e.sum(-1, keepdim=True)
    row = (top + torch.log(norm))[:, 0] - x.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    row = torch.where(counted, row, 0.0)
    member = (section[None] == torch.arange(1, case["k"] + 1, device="cuda")[:, None]) & counted[None]
    count = member.sum(-1)
    parts = (member * row.double()).sum(-1) / count.clamp(min=1)
    weights = torch.tensor(s["weights"], device="cuda", dtype=torch.float64)
    res = {"loss": (parts * weights).sum().float(), "parts": parts.float(), "rows": row}
    if case["grad"]:
        w = (weights / count.clamp(min=1) * case["scale"]).float()[section - 1] * counted
        d = e.div_(norm)
        d.scatter_add_(1, labels.clamp(min=0)[:, None], torch.full_like(norm, -1.0))
        s["d_logits"].copy_(d.mul_(w[:, None]))
        res["d_logits"] = s["d_logits"]
    return res


# --------------------------------------------------------------------------
# run
# --------------------------------------------------------------------------

def _run_own(s):
    from paper_2504_18583_amd import binding as B
    case = s["case"]
    if case["kind"] == "rope":
        how = dict(layout=case["layout"], q_gain=s["gq"], k_gain=s["gk"], eps=s["eps"])
        if not case["grad"]:
            q, k = B.qk_rope(s["q"], s["k"], s["pos"], s["table"], **how)
            return {"q": q, "k": k}
        dq, dk, dgq, dgk = B.qk_rope_grad(s["dq"], s["dk"], s["pos"], s["table"], q=s["q"], k=s["k"], **how)
        return {"dq": dq, "dk": dk} | ({"dgq": dgq, "dgk": dgk} if case["norm"] else {})
    if case["kind"] == "loss":
        loss, parts, by_row, d_logits = B.cod_loss(s["logits"], s["labels"], s["section"], case["k"],
                                                   weights=s["weights"], grad_scale=case["scale"],
                                                   d_logits=s["d_logits"], grad=case["grad"])
        return {"loss": loss, "parts": parts, "rows": by_row} | ({"d_logits": d_logits} if case["grad"] else {})
    out, lse = B.cod_attn(s["q"], s["k"], s["v"], s["plan"], s["scale"])
    res = {"out": out, "lse": lse}
    if case["train"]:
        res["dq"], res["dk"], res["dv"] = B.cod_attn_grad(s["d_out"], s["q"], s["k"], s["v"], out, lse, s["plan"],
                                                          s["scale"])
    return res


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "attn":
        return _attn_plain(s)
    if case["kind"] == "loss":
        return _loss_plain(s)
    if not case["grad"]:
        return {"q": _rope_plain(s["q"], s["gq"], s), "k": _rope_plain(s["k"], s["gk"], s)}
    dq, dgq = _rope_grad_plain(s["dq"], s["q"], s["gq"], s)
    dk, dgk = _rope_grad_plain(s["dk"], s["k"], s["gk"], s)
    return {"dq": dq, "dk": dk} | ({"dgq": dgq, "dgk": dgk} if case["norm"] else {})


# --------------------------------------------------------------------------
# work
# --------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rope":
        n = case["rows"] * (case["hq"] + case["hk"]) * case["hd"]
        table = min(case["rows"], case["max_pos"]) * case["rot"] * 4
        passes = 3 if case["grad"] and case["norm"] else 2     # the gradient of a norm reads its input too
        return {"bytes": float(passes * n * size + table + 4 * case["rows"]), "flops": 8.0 * n * (passes - 1)}
    if case["kind"] == "loss":
        n = case["rows"] * case["vocab"]
        return {"bytes": float(n * size * (2 if case["grad"] else 1) + 12 * case["rows"]), "flops": 4.0 * n}
    pairs = rows = 0.0
    for tokens in _lengths(case):
        n = tokens - 1
        kept = _keep_counts(n, case["k"])
        rows += sum(kept)
        # row (k, j) sees j - k + 2 real tokens and its k - 1 masks; kept columns are spread evenly
        pairs += sum(c * (n - k) / 2 + c * k for k, c in enumerate(kept, start=1))
    hq, hk, hd = case["hq"], case["hk"], case["hd"]
    heads = hq + hk                                            # one tensor of query heads, one of key heads: rows of each
    n_bytes = rows * hd * size * 2 * heads + rows * hq * 4
    flops = 4.0 * pairs * hd * hq
    if case["train"]:                                          # d_out in, dq, dk, dv out; five products
        n_bytes += rows * hd * size * 2 * heads
        flops += 10.0 * pairs * hd * hq
    return {"bytes": float(n_bytes), "flops": float(flops)}


# --------------------------------------------------------------------------
# exact: the definitions in float64
# --------------------------------------------------------------------------

def _rope_exact(x, gain, s, w, m, eps):
    """Rotation as a complex product, the norm in float64."""
    case = s["case"]
    y = x.double()
    if gain is not None:
        y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / y.shape[-1] + eps) * gain.double()
    half = case["rot"] // 2
    angle = s["pos"].double()[:, None, None] * w
    turn = torch.complex(torch.cos(angle) * m, torch.sin(angle) * m)
    if case["layout"] == "half":
        z = torch.complex(y[..., :half].contiguous(), y[..., half:2 * half].contiguous()) * turn
        return torch.cat([z.real, z.imag, y[..., 2 * half:]], -1)
    z = torch.view_as_complex(y[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * turn
    return torch.cat([torch.view_as_real(z).flatten(-2), y[..., 2 * half:]], -1)


def _attn_exact(s):
    case = s["case"]
    rows, hq, hd = s["q"].shape
    group = hq // s["k"].shape[1]
    res = {"out": torch.zeros(rows, hq, hd, device="cuda", dtype=torch.float64),
           "lse": torch.full((hq, rows), -math.inf, device="cuda", dtype=torch.float64)}
    if case["train"]:
        res |= {"d" + n: torch.zeros(s[n].shape, device="cuda", dtype=torch.float64) for n in "qkv"}
    for i, n in enumerate(s["lens"].tolist()):
        at = int(s["offsets"][i])
        sl = slice(at, at + n)
        k_of, j_of = s["section"][sl].long(), s["column"][sl].long()
        ka, ja, kb, jb = k_of[:, None], j_of[:, None], k_of[None], j_of[None]
        hidden = ~torch.where(kb == 1, jb <= ja - ka + 1, (kb <= ka) & (jb - kb == ja - ka))
        for h in range(hq):
            q, k, v = (s[t][sl, x].double().requires_grad_(case["train"]) for t, x in
                       (("q", h), ("k", h // group), ("v", h // group)))
            sc = torch.matmul(q, k.T).mul(s["scale"]).masked_fill_(hidden, -math.inf)
            lse = torch.logsumexp(sc.detach(), -1)
            out = torch.matmul(torch.exp(sc - lse[:, None]) if not case["train"] else torch.softmax(sc, -1), v)
            res["out"][sl, h], res["lse"][h, sl] = out.detach(), lse
            if case["train"]:
                grads = torch.autograd.grad(out, (q, k, v), s["d_out"][sl, h].double())
                for name, head, d in zip(("dq", "dk", "dv"), (h, h // group, h // group), grads):
                    res[name][sl, head] += d
            del sc, out
    return res


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        w, m = _inverse_frequencies(case)
        w = torch.from_numpy(w).cuda()
        if not case["grad"]:
            return {n: _rope_exact(s[n], s["g" + n], s, w, m, s["eps"]) for n in "qk"}
        res, gains = {}, {}
        for n in "qk":
            x = s[n].double().requires_grad_(True)
            g = None if s["g" + n] is None else s["g" + n].double().requires_grad_(True)
            d = torch.autograd.grad(_rope_exact(x, g, s, w, m, s["eps"]), (x,) if g is None else (x, g),
                                    s["d" + n].double())
            res["d" + n] = d[0]
            if g is not None:
                gains["dg" + n] = d[1]
        return res | gains
    if case["kind"] == "attn":
        return _attn_exact(s)
    # the loss, some rows at a time
    rows, k_max = case["rows"], case["k"]
    labels, section = s["labels"].long(), s["section"].long()
    counted = labels >= 0
    count = torch.bincount(section[counted], minlength=k_max + 1)[1:k_max + 1].clamp(min=1).double()
    weights = torch.tensor(s["weights"], device="cuda", dtype=torch.float64)
    total = torch.zeros(k_max + 1, device="cuda", dtype=torch.float64)
    by_row = torch.zeros(rows, device="cuda", dtype=torch.float64)
    d_logits = torch.zeros(rows, case["vocab"], device="cuda", dtype=torch.float64) if case["grad"] else None
    step = max(1, 200_000_000 // case["vocab"])
    for a in range(0, rows, step):
        b = slice(a, min(rows, a + step))
        logp = torch.log_softmax(s["logits"][b].double(), -1)
        pick = torch.nn.functional.one_hot(labels[b].clamp(min=0), case["vocab"]).bool()
        by_row[b] = torch.where(counted[b], -logp[pick], 0.0)
        total.index_add_(0, section[b], by_row[b])
        if case["grad"]:
            w = (weights / count)[section[b] - 1] * case["scale"] * counted[b]
            d_logits[b] = (logp.exp() - pick.double()) * w[:, None]
    parts = total[1:] / count
    return {"loss": (parts * weights).sum(), "parts": parts, "rows": by_row} | ({"d_logits": d_logits} if case["grad"] else {})
