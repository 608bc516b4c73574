"""Bounds of float16 attention: small beside what they bound, and held by the
computation that they are derived for."""
import numpy as np
import pytest
import torch

import serve_bounds as SB
import serve_common as S


def _case(rows, past, hq, hk, hd, window=0, sinks=0, std=1.0):
    g = torch.Generator().manual_seed(rows + past)
    batch = S.Batch([rows], [past], 16, window, sinks)
    n = rows + past
    K, V, q = (torch.randn(m, h, hd, generator=g).mul(s).half() for m, h, s in ((n, hk, std), (n, hk, 1.0), (rows, hq, std)))
    at = lambda x: lambda s, j: x[torch.as_tensor(j)].double()  # noqa: E731
    return batch, q, K, V, at(K), at(V)


@pytest.mark.parametrize("rows,past,hd", [(1, 511, 128), (2, 1500, 64), (1, 4000, 128), (9, 9000, 64), (1, 20000, 128)])
def test_bounds_are_small_beside_the_output(rows, past, hd):
    batch, q, _, _, k_of, v_of = _case(rows, past, 2, 1, hd)
    out, bound = SB.sharp_attn_ref(q, k_of, v_of, batch, hd ** -0.5)["out"]
    rms = float(out.square().mean().sqrt())
    assert float(bound.median()) < rms / 6 and float(bound.max()) < rms / 3, (float(bound.median()), float(bound.max()), rms)


@pytest.mark.parametrize("rows,past,hd,window,sinks,std", [(3, 2000, 64, 0, 0, 1.0), (2, 5000, 128, 0, 0, 1.0), (20, 700, 64, 100, 5, 1.0),
                                                           (4, 900, 64, 0, 0, 4.0), (1, 0, 64, 0, 0, 1.0)])
def test_bounds_hold_for_the_rounded_computation(rows, past, hd, window, sinks, std):
    """Probabilities under a maximum that runs up to 2^8 behind, rounded to float16
    with its subnormal steps, stages of 64 keys."""
    batch, q, K, V, k_of, v_of = _case(rows, past, 2, 1, hd, window, sinks, std)
    scale = hd ** -0.5
    out, bound = SB.sharp_attn_ref(q, k_of, v_of, batch, scale)["out"]
    j, seen = batch.seen(0)
    k, v = k_of(0, j)[:, 0], v_of(0, j)[:, 0]
    lost = 0
    for h in range(2):
        sc = (q[:, h].double() @ k.T * scale).masked_fill(~seen, -np.inf) / np.log(2)
        m, l, o = torch.full((rows,), -1e30, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, hd, dtype=torch.float64)
        for at in range(0, len(j), 64):
            s = sc[:, at:at + 64]
            top = s.amax(-1)
            new = torch.where(top > m + 8, top, m)
            f = torch.exp2(m - new)
            m, l, o = new, l * f, o * f[:, None]
            p = torch.exp2(s - m[:, None])
            lost += int((p.half().double() != p).logical_and(p < 2.0 ** -14).sum())
            l, o = l + p.sum(-1), o + p.half().double() @ v[at:at + 64]
        got = (o / l[:, None]).half().double()
        assert bool(((got - out[:, h]).abs() <= bound[:, h]).all())
    assert lost or std < 4                           # (peaked rows have subnormal probabilities)
