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
