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
