"""GPU checks of the mask-token training operators at the ends of what their
documentation allows: the most rows, no epsilon, the longest sample, padded
batches."""
import numpy as np
import pytest
import torch

import train_common as T
from gpu_common import require_gpu, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    require_gpu()
    from paper_2504_18583_amd import binding
    return binding


def _randn(gen, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("rows", [2 ** 31 - 1, 2 ** 31 - 48])
def test_rope_of_the_most_rows(B, rows):
    """Row numbers up to the last that 32 bits hold: every row's bits are those of
    the same rows in a call of 2^24."""
    chunk, hd = 1 << 24, 8
    g = _gen(rows % 1000)
    table, gain = B.rope_table(64, hd, 1e4), 1 + _randn(g, hd, std=0.1)
    base, dy = (_randn(g, chunk, 1, hd, dtype=torch.bfloat16) for _ in range(2))
    base_pos = torch.randint(0, 64, (chunk,), generator=g, device="cuda", dtype=torch.int32)

    def spread(t, out):
        for a in range(0, rows, chunk):
            out[a:a + chunk].copy_(t[:min(chunk, rows - a)])
        return out

    def check(got, want, what):
        for a in range(0, rows, chunk):
            n = min(chunk, rows - a)
            assert torch.equal(got[a:a + n], want[:n]), (what, a)
    pos = spread(base_pos, torch.empty(rows, dtype=torch.int32, device="cuda"))
    x, d = (torch.empty(rows, 1, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for norm in (None, gain):
        say(f"[gpu] rope of {rows} rows, norm={norm is not None}")
        want, _ = B.qk_rope(base, None, base_pos, table, q_gain=norm)
        spread(base, x)
        B.qk_rope(x, None, pos, table, q_gain=norm, q_out=x)
        check(x, want, "forward")
        want, _, _, _ = B.qk_rope_grad(dy, None, base_pos, table, q=base, q_gain=norm)
        spread(base, x)
        spread(dy, d)
        _, _, dg, _ = B.qk_rope_grad(d, None, pos, table, q=x, q_gain=norm, q_dx=d)
        check(d, want, "gradient")
        assert norm is None or dg.isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", [(77, 32, 8, 128, 128), (5, 2, 1, 64, 64), (300, 2, 1, 64, 32), (41, 5, 1, 80, 40), (9, 3, 2, 24, 8),
                                   (33, 3, 0, 64, 64), (7, 4, 2, 256, 128), (6, 3, 1, 34, 34)], ids=str)
def test_rope_norm_without_epsilon(B, shape, layout, dtype):
    """eps = 0 and no head of zeros: finite sums, also where the heads are no
    multiple of those that a workgroup takes together."""
    rows, hq, hk, hd, rot = shape
    g, dt = _gen(rows + hd), T.DTYPES[dtype]
    say(f"[gpu] rope without epsilon {shape} {layout} {dtype}")
    table = B.rope_table(50, rot, 1e4)
    pos = torch.randint(0, 50, (rows,), generator=g, device="cuda", dtype=torch.int32)
    q, dq = (_randn(g, rows, hq, hd, dtype=dt) for _ in range(2))
    k, dk = (_randn(g, rows, hk, hd, dtype=dt) if hk else None for _ in range(2))
    gq, gk = 1 + _randn(g, hd, std=0.2), 1 + _randn(g, hd, std=0.2) if hk else None
    yq, yk = B.qk_rope(q, k, pos, table, layout, gq, gk, eps=0.0)
    xq, xk, gdq, gdk = B.qk_rope_grad(dq, dk, pos, table, layout, q, k, gq, gk, eps=0.0)
    for name, x, y, gain, dy, dx, dg in (("q", q, yq, gq, dq, xq, gdq), ("k", k, yk, gk, dk, xk, gdk)):
        if x is None:
            continue
        T.assert_within(y, *T.rope_ref(x, pos, table, layout, gain, 0.0), name)
        want, bound, want_g, bound_g = T.rope_grad_ref(dy, x, pos, table, layout, gain, 0.0)
        T.assert_within(dx, want, bound, f"d{name}")
        T.assert_within(dg, want_g, bound_g, f"d{name} gain")


def test_attention_and_rotation_in_autograd(B):
    """The calls inside autograd Functions: their gradients, bit for bit, and in
    place of a graph without them an error."""
    section, column, offs, lens, rows = T.pack([40, 9], 4)
    plan = B.cod_plan(torch.from_numpy(section).cuda(), torch.from_numpy(column).cuda(), offs, torch.from_numpy(lens).cuda())
    table, pos = B.rope_table(64, 64, 1e4), torch.from_numpy(column).cuda()
    g = _gen(5)

    class Rotated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, gq, gk):
            ctx.save_for_backward(q, k, gq, gk)
            return B.qk_rope(q, k, pos, table, q_gain=gq, k_gain=gk)

        @staticmethod
        def backward(ctx, dq, dk):
            q, k, gq, gk = ctx.saved_tensors
            return B.qk_rope_grad(dq, dk, pos, table, q=q, k=k, q_gain=gq, k_gain=gk)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            out, lse = B.cod_attn(q, k, v, plan)
            ctx.save_for_backward(q, k, v, out, lse)
            return out

        @staticmethod
        def backward(ctx, d_out):
            return B.cod_attn_grad(d_out, *ctx.saved_tensors, plan)

    q, k, v = (_randn(g, rows, h, 64, dtype=torch.bfloat16).requires_grad_() for h in (4, 2, 2))
    gq, gk = (1 + _randn(g, 64, std=0.1) for _ in range(2))
    gq.requires_grad_(), gk.requires_grad_()
    with pytest.raises(B.PardError, match="autograd.Function"):
        B.cod_attn(q, k, v, plan)
    with pytest.raises(B.PardError, match="autograd.Function"):
        B.qk_rope(q.detach(), k.detach(), pos, table, q_gain=gq, k_gain=gk)
    d_out = _randn(g, rows, 4, 64, dtype=torch.bfloat16)
    rq, rk = Rotated.apply(q, k, gq, gk)
    Attention.apply(rq, rk, v).backward(d_out)
    with torch.no_grad():
        sq, sk = B.qk_rope(q, k, pos, table, q_gain=gq, k_gain=gk)
        out, lse = B.cod_attn(sq, sk, v, plan)
        dq, dk, dv = B.cod_attn_grad(d_out, sq, sk, v, out, lse, plan)
        want = (*B.qk_rope_grad(dq, dk, pos, table, q=q, k=k, q_gain=gq, k_gain=gk), dv)
    for got, w in zip((q.grad, k.grad, gq.grad, gk.grad, v.grad), want):
        assert torch.equal(got, w)


def _attn_rows(q, k, v, d_out, section, column, rows, scale):
    """Attention of one sample in float64 on the device, for the queries `rows`
    alone: (value, bound) of out, lse and dq [len(rows), ..], and of dk and dv as
    those rows add to them.  Bounds as train_common.attn_ref counts them."""
    hq, hk = q.shape[1], k.shape[1]
    u, F = T.unit(q.dtype), T.F
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device="cuda")  # noqa: E731
    n, hd = len(rows), q.shape[2]
    res = {name: (z(n, hq, hd), z(n, hq, hd)) for name in ("out", "dq")} | {"lse": (z(hq, n), z(hq, n))}
    res |= {name: (z(*k.shape), z(*k.shape)) for name in ("dk", "dv")}
    chain = column - section
    for a in range(0, n, 512):
        sl = slice(a, min(a + 512, n))
        r = rows[sl]
        ka, ja = section[r][:, None], column[r][:, None]
        seen = torch.where(section == 1, column <= ja - ka + 1, (section <= ka) & (chain == ja - ka))
        terms = int(seen.sum(-1).max())
        for h in range(hq):
            g = h * hk // hq
            Q, G, K, V = q[r, h].double(), d_out[r, h].double(), k[:, g].double(), v[:, g].double()
            KT, VT = K.T.contiguous(), V.T.contiguous()
            sc = (Q @ KT * scale).masked_fill_(~seen, -np.inf)
            lse = torch.logsumexp(sc, -1)
            P = torch.exp(sc - lse[:, None])
            out, A = P @ V, P @ V.abs()
            ds_max = ((Q.abs() @ KT.abs() * abs(scale)) * seen).amax(-1) * (hd + 8) * F
            rel = 2 * ds_max[:, None] + (terms + 32) * F
            e_out = u * (A + out.abs()) + A * rel
            res["out"][0][sl, h], res["out"][1][sl, h] = out, e_out
            res["lse"][0][h, sl], res["lse"][1][h, sl] = lse, ds_max + (terms + 16) * F + 4 * F * lse.abs()
            delta = (G * out).sum(-1, keepdim=True)
            e_delta = (G.abs() * e_out).sum(-1, keepdim=True) + hd * F * (G.abs() * out.abs()).sum(-1, keepdim=True)
            dS = P * (G @ VT - delta)
            e_dS = (u * dS.abs() + P * e_delta + 2 * rel * P * (G.abs() @ VT.abs() + delta.abs())) * seen
            e_P = P * (u + 2 * rel) * seen
            sums = (n * hq // hk + terms) * F
            dq, mag = scale * dS @ K, abs(scale) * dS.abs() @ K.abs()
            res["dq"][0][sl, h], res["dq"][1][sl, h] = dq, abs(scale) * e_dS @ K.abs() + sums * mag + u * dq.abs()
            for name, m, e, x, f in (("dk", dS, e_dS, Q, scale), ("dv", P, e_P, G, 1.0)):
                res[name][0][:, g] += f * (m.T.contiguous() @ x)
                res[name][1][:, g] += abs(f) * ((e + sums * m.abs()).T.contiguous() @ x.abs())
    for name in ("dk", "dv"):
        res[name][1].add_(u * res[name][0].abs())
    return res


def _check_rows(B, section, column, heads, hd, rows, keys):
    """One sample, its rows in `rows` and keys in `keys` (seen by no others than
    `rows`), and a second short sample behind it."""
    hq, hk = heads
    s2, c2, _, _, n2 = T.pack([21], 4)
    n = len(section)
    sec, col = (torch.from_numpy(np.concatenate(x).astype(np.int32)).cuda() for x in ((section, s2), (column, c2)))
    plan = B.cod_plan(sec, col, [0, n, n + n2], torch.tensor([n, n2], dtype=torch.int32, device="cuda"))
    g = _gen(n)
    q, d_out = (_randn(g, n + n2, hq, hd, dtype=torch.bfloat16) for _ in range(2))
    k, v = (_randn(g, n + n2, hk, hd, dtype=torch.bfloat16) for _ in range(2))
    say(f"[gpu] attention: {n} rows of one sample, {hq}/{hk} heads x {hd}")
    out, lse = B.cod_attn(q, k, v, plan)
    dq, dk, dv = B.cod_attn_grad(d_out, q, k, v, out, lse, plan)
    got = {"out": out[rows], "lse": lse[:, rows], "dq": dq[rows], "dk": dk[keys], "dv": dv[keys]}
    ref = _attn_rows(q[:n], k[:n], v[:n], d_out[:n], sec[:n].long(), col[:n].long(), rows, hd ** -0.5)
    for name, (want, bound) in ref.items():
        pick = keys if name in ("dk", "dv") else slice(None)
        T.assert_within(got[name], want[pick].cpu(), bound[pick].cpu(), name)
    want = T.attn_ref(q[n:], k[n:], v[n:], s2, c2, np.array([0, n2]), [n2], hd ** -0.5, d_out[n:])
    for name, x in (("out", out[n:]), ("lse", lse[:, n:]), ("dq", dq[n:]), ("dk", dk[n:]), ("dv", dv[n:])):
        T.assert_within(x, *want[name], f"{name} of the sample behind")


@pytest.mark.parametrize("heads,hd", [((2, 1), 64), ((1, 1), 128)])
def test_attention_of_the_longest_sample(B, heads, hd):
    """8192 columns: every row and key."""
    section, column, _, _, n = T.pack([8192], 8)
    rows = torch.arange(n, device="cuda")
    _check_rows(B, section, column, heads, hd, rows, rows)


def test_attention_of_the_largest_sample(B):
    """8192 columns of which 64 subtasks keep everything, 522 272 rows: rows of
    the first, some middle and the last chains, and the keys that only they see."""
    section = np.concatenate([np.full(8192 - k + 1, k) for k in range(1, 65)])
    column = np.concatenate([np.arange(k - 1, 8192) for k in range(1, 65)])
    chain = torch.from_numpy(column - section + 1).cuda()
    picked = torch.isin(chain, torch.tensor([0, 1, 127, 4096, 8191 - 63, *range(8186, 8192)], device="cuda"))
    rows = picked.nonzero()[:, 0]
    late = (chain >= 8186) | (picked & (torch.from_numpy(section).cuda() > 1))
    _check_rows(B, section, column, (2, 1), 64, rows, late.nonzero()[:, 0])


def test_more_columns_than_a_sample_may_have(B):
    n = 8193
    section = torch.ones(n, dtype=torch.int32, device="cuda")
    column = torch.arange(n, dtype=torch.int32, device="cuda")
    for m in (n, 8192):
        length = torch.tensor([m], dtype=torch.int32, device="cuda")
        if m == 8192:
            B.cod_plan(section, column, [0, n], length)
            continue
        with pytest.raises(B.PardError) as e:
            B.cod_plan(section, column, [0, n], length)
        assert e.value.status == B.PARD_ERR_ARG


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "f16")])
def test_attention_gradient_again(B, hd, dtype):
    """A second gradient of the same tensors gives the same bits."""
    section, column, offs, lens, rows = T.pack([130, 60, 700], 8)
    plan = B.cod_plan(torch.from_numpy(section).cuda(), torch.from_numpy(column).cuda(), offs, torch.from_numpy(lens).cuda())
    g = _gen(6)
    q, k, v, d_out = (_randn(g, rows, h, hd, dtype=T.DTYPES[dtype]) for h in (4, 2, 2, 4))
    out, lse = B.cod_attn(q, k, v, plan)
    first = B.cod_attn_grad(d_out, q, k, v, out, lse, plan)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, B.cod_attn_grad(d_out, q, k, v, out, lse, plan)))


def test_a_padded_batch(B):
    """Regions longer than their samples, whose last rows hold anything: with
    ids, positions and labels cleared there, nothing of them reaches the loss or a
    gradient, the gains' among them."""
    k_max, hd, vocab, dt = 5, 64, 300, torch.bfloat16
    rng = np.random.default_rng(3)
    lengths = [2, 30, 7, 111]
    token_offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    tokens = torch.from_numpy(rng.integers(0, vocab - 1, size=int(token_offsets[-1])).astype(np.int32)).cuda()
    offsets, data, lens = B.cod_build(tokens, token_offsets, k_max, 1.0, 0.2, vocab - 1, 9)
    inside = torch.cat([torch.arange(b - a, device="cuda") < n for a, b, n in zip(offsets, offsets[1:], lens)])
    assert not inside.all()
    g = _gen(11)
    emb, w = _randn(g, vocab, 8 * hd, dtype=dt), _randn(g, 4 * hd, vocab, dtype=dt, std=0.05)
    gq, gk, table = 1 + _randn(g, hd, std=0.1), 1 + _randn(g, hd, std=0.1), B.rope_table(128, hd, 1e4)
    want = None
    for anything in (0, -1, 2 ** 31 - 1, -2 ** 31):
        say(f"[gpu] a padded batch, {anything} past the samples")
        rows = {name: t.masked_fill(~inside, anything) for name, t in data.items()}
        ids, labels, pos = (rows[name].masked_fill(~inside, x) for name, x in (("ids", 0), ("labels", -1), ("pos", 0)))
        plan = B.cod_plan(rows["section"], rows["column"], offsets, lens)
        q, k, v = (t.unflatten(1, (-1, hd)) for t in emb[ids.long()].split((4 * hd, 2 * hd, 2 * hd), 1))
        rq, rk = B.qk_rope(q, k, pos, table, q_gain=gq, k_gain=gk)
        out, lse = B.cod_attn(rq, rk, v, plan)
        loss, parts, by_row, d_logits = B.cod_loss(out.flatten(1) @ w, labels, rows["section"], k_max, grad_scale=64.0)
        d_out = (d_logits @ w.T.contiguous()).unflatten(1, (4, hd))
        dq, dk, dv = B.cod_attn_grad(d_out, rq, rk, v, out, lse, plan)
        got = (loss, parts, by_row, dv, *B.qk_rope_grad(dq, dk, pos, table, q=q, k=k, q_gain=gq, k_gain=gk))
        assert all(t.isfinite().all() for t in got)
        assert all((t[~inside] == 0).all() for t in got[2:6])
        assert got[6].abs().max() > 0 and got[7].abs().max() > 0
        want = want or got
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_optional_outputs_and_shared_inputs(B):
    """The C calls without lse and row_loss; inputs whose key heads, rows of
    queries or gradients' rows are one and the same (stride 0)."""
    section, column, offs, lens, rows = T.pack([50, 3], 4, slack=2)
    plan = B.cod_plan(torch.from_numpy(section).cuda(), torch.from_numpy(column).cuda(), offs, torch.from_numpy(lens).cuda())
    g = _gen(8)
    q, v = _randn(g, rows, 4, 64, dtype=torch.bfloat16), _randn(g, rows, 2, 64, dtype=torch.bfloat16)
    k, d_out = _randn(g, rows, 1, 64, dtype=torch.bfloat16).expand(rows, 2, 64), _randn(g, 1, 4, 64, dtype=torch.bfloat16).expand(rows, 4, 64)
    assert k.stride(1) == d_out.stride(0) == 0
    say("[gpu] attention of shared inputs")
    out, lse = B.cod_attn(q, k, v, plan)
    dq, dk, dv = B.cod_attn_grad(d_out, q, k, v, out, lse, plan)
    want = T.attn_ref(q, k, v, section, column, offs, lens, 64 ** -0.5, d_out)
    inside = torch.cat([torch.arange(b - a) < n for a, b, n in zip(offs, offs[1:], lens)])
    for name, x in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
        T.assert_within(x[inside.cuda()], want[name][0][inside], want[name][1][inside], name)
    again = torch.zeros_like(out)
    args = B.pard_cod_attn_args(B.C.pointer(plan.plan), 4, 2, 64, B.PARD_BF16, 64 ** -0.5)
    heads = [B.pard_heads(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, k, v, again)]
    stream = torch.cuda.current_stream().cuda_stream
    assert B.lib.pard_cod_attn(args, *heads, None, stream) == B.PARD_OK
    assert torch.equal(again, out)

    table, pos = B.rope_table(64, 64, 1e4), torch.from_numpy(np.clip(column, 0, 63)).cuda()
    one = _randn(g, 1, 2, 64).expand(rows, 2, 64)
    y, _ = B.qk_rope(one, None, pos, table)
    T.assert_within(y, *T.rope_ref(one, pos, table, "half", None, 1e-6), "rotation of one row")

    logits = _randn(g, 20, 1000)
    labels = torch.arange(20, dtype=torch.int32, device="cuda")
    loss, parts, _, d = B.cod_loss(logits, labels, None, 1)
    d2, loss2 = torch.empty_like(logits), torch.empty(2, device="cuda")
    a = B.pard_cod_loss_args(20, 1000, B.PARD_F32, 1, 1.0, logits.data_ptr(), 1000, labels.data_ptr(), None, None, d2.data_ptr(), 1000,
                             loss2.data_ptr(), None)
    n = B.lib.pard_cod_loss_workspace_bytes(a)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert B.lib.pard_cod_loss(a, ws.data_ptr(), n, stream) == B.PARD_OK
    assert torch.equal(d, d2) and torch.equal(loss2, torch.stack([loss, parts[0]]))
