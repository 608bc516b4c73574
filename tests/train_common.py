"""Plain float64 forms of the mask-token training operators, with the bounds
that their GPU results are held to.

u = eps / 2 is a rounding of the stored type (half a unit in the last place),
F = 2^-24 one of float32.  Bounds add up what a float32 computation of the
formula may be off, in any order of its sums (n terms: n F times the sum of
their magnitudes), and the roundings to the stored type."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cod

F = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def unit(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def floor_of(dtype) -> float:
    """Half the smallest subnormal step where it matters (float16)."""
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


def assert_within(got, want, bound, what):
    got = got.detach().double().cpu()
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; first at {i}: {got[i]} for {want[i]} "
                             f"(bound {bound[i]:.3g}); worst ratio {float(((got - want).abs() / bound.clamp(min=1e-300)).max()):.3g}")


# ---- rotary positions -------------------------------------------------------

def turn(x, cos, sin, layout):
    h = cos.shape[-1]
    if layout == "half":
        a, b = x[..., :h], x[..., h:2 * h]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * h:]], -1)
    a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., 2 * h:]], -1)


def rope_ref(x, pos, table, layout, gain, eps):
    """(y, bound) in float64 from the float32 table."""
    dt, x = x.dtype, x.double().cpu()
    cs = table.double().cpu()[pos.long().cpu()][:, None]
    n = x
    if gain is not None:
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    y = turn(n, cs[..., 0], cs[..., 1], layout)
    mag = turn(n.abs(), cs[..., 0].abs(), -cs[..., 1].abs(), layout).abs() + turn(n.abs(), cs[..., 0].abs(), cs[..., 1].abs(), layout).abs()
    # r: hd roundings of the sum of squares (halved by the root) and 4 more, two
    # products, then two products and a sum
    terms = 4 + (0 if gain is None else x.shape[-1] / 2 + 8)
    return y, unit(dt) * y.abs() + terms * F * mag + floor_of(dt)


def rope_grad_ref(dy, x, pos, table, layout, gain, eps):
    """(dx, bound, dgain, bound)"""
    dt, dy = dy.dtype, dy.double().cpu()
    cs = table.double().cpu()[pos.long().cpu()][:, None]
    dn = turn(dy, cs[..., 0], -cs[..., 1], layout)
    mag = turn(dy.abs(), cs[..., 0].abs(), cs[..., 1].abs(), layout).abs() + turn(dy.abs(), cs[..., 0].abs(), -cs[..., 1].abs(), layout).abs()
    if gain is None:
        return dn, unit(dt) * dn.abs() + 4 * F * mag + floor_of(dt), None, None
    x, g = x.double().cpu(), gain.double().cpu()
    hd = x.shape[-1]
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh, t = x * r, dn * g
    mean = (t * xh).mean(-1, keepdim=True)
    dx = r * (t - xh * mean)
    mag_t = mag * g.abs()
    mag_dx = r * (mag_t + xh.abs() * (mag_t * xh.abs()).mean(-1, keepdim=True))
    terms = 2 * hd + 24
    dg, mag_g = (dn * xh).sum((0, 1)), (mag * xh.abs()).sum((0, 1))
    n = x.shape[0] * x.shape[1]
    return dx, unit(dt) * dx.abs() + terms * F * mag_dx + floor_of(dt), dg, (n + hd / 2 + 24) * F * mag_g + 1e-30


# ---- packed rows and attention ---------------------------------------------

def pack(lengths, k_max, r=0.7, r_min=0.2, seed=3, slack=0, lead=0, trail=0):
    """Packed samples of the oracle: section, column (int32), out_offsets, lens;
    regions `slack` rows larger, `lead` rows before and `trail` after them."""
    parts = [cod.cod_process(list(range(n + 1)), k_max, r, r_min, 0, seed, i) if n else None
             for i, n in enumerate(lengths)]
    lens = [len(p.ids) if p else 0 for p in parts]
    offs = lead + np.concatenate([[0], np.cumsum([n + slack for n in lens])]).astype(np.int64)
    rows = int(offs[-1]) + trail
    section, column = np.full(rows, 77, np.int32), np.full(rows, -5, np.int32)   # (rows of no sample: anything)
    for p, o, n in zip(parts, offs, lens):
        if p:
            section[o:o + n], column[o:o + n] = p.section, p.column
    return section, column, offs, np.array(lens, np.int32), rows


def seen_mask(section, column):
    """[rows, rows]: whether a row attends to another (one sample)."""
    k, j = torch.as_tensor(section).long(), torch.as_tensor(column).long()
    ka, ja, kb, jb = k[:, None], j[:, None], k[None], j[None]
    return torch.where(kb == 1, jb <= ja - ka + 1, (kb <= ka) & (jb - kb == ja - ka))


def attn_ref(q, k, v, section, column, offs, lens, scale, d_out=None):
    """Dict of (value, bound) in float64: out, lse and, with d_out, dq, dk, dv,
    of the rows in samples; other rows hold 0 with bound 0 (lse -inf)."""
    dt = q.dtype
    rows, hq, hd = q.shape
    hk = k.shape[1]
    group = hq // hk
    q, k, v = (t.double().cpu() for t in (q, k, v))
    z = lambda like: torch.zeros(like.shape, dtype=torch.float64)  # noqa: E731
    res = {"out": (z(q), z(q)), "lse": (torch.full((hq, rows), -np.inf, dtype=torch.float64), torch.zeros(hq, rows, dtype=torch.float64))}
    if d_out is not None:
        d_out = d_out.double().cpu()
        res |= {n: (z(t), z(t)) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    u, fl = unit(dt), floor_of(dt)
    for o, n in zip(offs[:-1], lens):
        sl = slice(int(o), int(o) + int(n))
        if n == 0:
            continue
        seen = seen_mask(section[sl], column[sl])
        for h in range(hq):
            g = h // group
            Q, K, V = q[sl, h], k[sl, g], v[sl, g]
            sc = (Q @ K.T * scale).masked_fill(~seen, -np.inf)
            lse = torch.logsumexp(sc, -1)
            P = torch.exp(sc - lse[:, None])
            out = P @ V
            # a score's error: hd terms of its product (fp32), the scale and the
            # exponent's argument (scores in base 2, up to their magnitude)
            ds_max = ((Q.abs() @ K.abs().T * abs(scale)) * seen).amax(-1) * (hd + 8) * F
            rel = 2 * ds_max[:, None] + (n + 32) * F
            A = P @ V.abs()
            e_out = u * (A + out.abs()) + A * rel + fl * (1 + n * 256 * V.abs().amax())
            res["out"][0][sl, h], res["out"][1][sl, h] = out, e_out
            res["lse"][0][h, sl] = lse
            res["lse"][1][h, sl] = ds_max + (n + 16) * F + 4 * F * lse.abs()
            if d_out is None:
                continue
            G = d_out[sl, h]
            dP = G @ V.T
            delta = (G * out).sum(-1, keepdim=True)
            dS = P * (dP - delta)
            # delta is formed from the rounded output
            e_delta = (G.abs() * e_out).sum(-1, keepdim=True) + hd * F * (G.abs() * out.abs()).sum(-1, keepdim=True)
            e_dS = u * dS.abs() + P * e_delta + 2 * rel * P * (G.abs() @ V.abs().T + delta.abs()) + fl
            e_P = P * (u + 2 * rel) + fl
            nq = group * n
            for name, row, val, err, mag in (
                    ("dq", (sl, h), scale * dS @ K, abs(scale) * (e_dS * seen) @ K.abs(), abs(scale) * dS.abs() @ K.abs()),
                    ("dk", (sl, g), scale * dS.T @ Q, abs(scale) * (e_dS * seen).T @ Q.abs(), abs(scale) * dS.abs().T @ Q.abs()),
                    ("dv", (sl, g), P.T @ G, (e_P * seen).T @ G.abs(), P.T @ G.abs())):
                res[name][0][row] += val
                res[name][1][row] += err + nq * F * mag
    for name in ("dq", "dk", "dv") if d_out is not None else ():
        res[name][1].add_(u * res[name][0].abs() + fl)
    return res


# ---- the loss ---------------------------------------------------------------

def loss_ref(logits, labels, section, n_sections, weights, grad_scale):
    """(loss, parts, rows, d_logits) in float64 and the bounds of the last two
    relative to their parts: row bound [rows], gradient bound."""
    dt = logits.dtype
    x = logits.double().cpu()
    rows, vocab = x.shape
    labels, section = labels.long().cpu(), section.long().cpu()
    counted = (labels >= 0) & (section >= 1) & (section <= n_sections)
    lab = labels.clamp(min=0)
    lse = torch.logsumexp(x, -1)
    row = torch.where(counted, lse - x[torch.arange(rows), lab], 0.0)
    count = torch.stack([((section == k) & counted).sum() for k in range(1, n_sections + 1)]).double()
    parts = torch.stack([row[(section == k) & counted].sum() for k in range(1, n_sections + 1)]) / count.clamp(min=1)
    if weights is None:
        loss = row.sum() / count.sum().clamp(min=1)
        w = counted.double() / count.sum().clamp(min=1)
    else:
        wt = torch.tensor(weights, dtype=torch.float64)
        loss = (parts * wt).sum()
        w = counted * (wt / count.clamp(min=1))[(section.clamp(1, n_sections) - 1)]
    w = w * grad_scale
    p = torch.softmax(x, -1)
    d = p.clone()
    d[torch.arange(rows), lab] -= 1
    d = d * w[:, None]
    # lse: vocab terms, the exponents' arguments up to the logits' magnitude
    top = x.abs().amax(-1)
    e_lse = (vocab ** 0.5 * 8 + 32 + 8 * top) * F
    e_row = torch.where(counted, e_lse + 4 * F * (lse.abs() + x[torch.arange(rows), lab].abs()), 0.0)
    onehot = torch.zeros_like(p)
    onehot[torch.arange(rows), lab] = 1
    e_d = unit(dt) * d.abs() + w.abs()[:, None] * (p * (2 * e_lse[:, None] + 16 * F + 8 * F * top[:, None]) + 4 * F * onehot) + floor_of(dt)
    e_d = torch.where(counted[:, None], e_d, 0.0)
    return loss, parts, row, d, e_row, e_d
