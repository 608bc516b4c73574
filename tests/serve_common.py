"""Plain float64 forms of the serving operators (a paged cache, attention over
it, logits before tokens are picked), with the bounds that their GPU results
are held to.  u, F and the way bounds add up are train_common's."""
from __future__ import annotations

import numpy as np
import torch

from train_common import DTYPES, F, floor_of, unit

BLOCK = 32
BITS = {"e4m3": (3, -6, 448.0), "e2m1": (1, 0, 6.0)}      # bits of the fraction, smallest normal exponent, largest value


def grid(cache):
    """Values of the codes without their sign, ascending (float64)."""
    bits, low, top = BITS[cache]
    n, out, e = 1 << bits, [], low
    out += [m / n * 2.0 ** low for m in range(n)]
    while out[-1] < top:
        out += [(1 + m / n) * 2.0 ** e for m in range(n)]
        e += 1
    return torch.tensor([v for v in out if v <= top], dtype=torch.float64)


def stored(x, cache):
    """float64 [..., n]: what the cache holds of x, block by block."""
    g = grid(cache)
    b = x.double().cpu().unflatten(-1, (-1, BLOCK))
    big = b.abs().amax(-1, keepdim=True)
    ok = torch.isfinite(b).all(-1, keepdim=True)
    b = torch.where(ok, b, 0.0)
    big = torch.where(ok, big, 0.0)
    scale = torch.full_like(big, 2.0 ** -126)
    while bool((big > g[-1] * scale).any()):
        scale = torch.where(big > g[-1] * scale, 2 * scale, scale)
    a = (b / scale).abs()
    hi = torch.searchsorted(g, a.contiguous()).clamp(max=len(g) - 1)
    lo = (hi - 1).clamp(min=0)
    near_hi, near_lo = g[hi] - a, a - g[lo]
    at = torch.where((near_hi < near_lo) | ((near_hi == near_lo) & (hi % 2 == 0)), hi, lo)
    return torch.where(ok, torch.copysign(g[at], b) * scale, float("nan")).flatten(-2)


def decoded(codes, scales, cache):
    """float64 values of a cache's bytes, by a table of its codes."""
    g, codes, scales = grid(cache), codes.cpu().long(), scales.cpu().long()
    if cache == "e4m3":
        t = torch.cat([g, torch.tensor([float("nan")], dtype=torch.float64)])
        v = torch.cat([t, -t])[codes]
    else:
        v = torch.cat([g, -g])[torch.stack([codes & 15, codes >> 4], -1).flatten(-2)]
    s = torch.where(scales == 255, float("nan"), torch.exp2(scales.double() - 127))
    return v * s.repeat_interleave(BLOCK, -1)


class Batch:
    """Sequences of a step on the host: rows[s] new rows after past[s] positions,
    pages in a random order with spare ones, `lead` rows before and `trail`
    behind them, table entries that no row needs garbage."""

    def __init__(self, rows, past, page, window=0, sinks=0, lead=0, trail=0, seed=0, spare=3, first_page=0):
        rng = np.random.default_rng(seed)
        self.rows, self.past, self.page = np.array(rows), np.array(past), page
        self.window, self.sinks = window, sinks
        need = -(-(self.rows + self.past) // page)
        self.n_pages = first_page + int(need.sum()) + spare
        order = first_page + rng.permutation(self.n_pages - first_page)
        self.width = int(need.max()) + 2
        garbage = np.array([-1, -(1 << 31), (1 << 31) - 1, self.n_pages, 0])
        self.table = garbage[rng.integers(0, 5, (len(rows), self.width))].astype(np.int32)
        self.row_start = (lead + np.concatenate([[0], np.cumsum(self.rows)])).astype(np.int32)
        self.n = int(self.row_start[-1]) + trail
        self.kv_len = (self.rows + self.past).astype(np.int32)
        at = 0
        for s, n in enumerate(need):
            if not self.rows[s]:
                continue
            first = max(past[s] - window + 1, 0) // page if window else 0
            for p in range(n):
                if p >= first or p * page < sinks:
                    self.table[s, p] = order[at + p]
            at += n

    def seq_rows(self, s):
        return range(int(self.row_start[s]), int(self.row_start[s + 1]))

    def places(self, s, positions):
        positions = np.asarray(positions)
        return torch.as_tensor(self.table[s, positions // self.page]).long(), torch.as_tensor(positions % self.page)

    def owned(self):
        m = torch.zeros(self.n, dtype=torch.bool)
        m[self.row_start[0]:self.row_start[-1]] = True
        return m

    def device(self, B, max_seq_rows=0):
        t = [torch.from_numpy(x).cuda() for x in (self.table, self.row_start, self.kv_len)]
        return B.KVBatch(*t, max_seq_rows=max_seq_rows)

    def seen(self, s):
        """(positions, mask [rows, positions]) of what sequence s's rows see."""
        p = self.past[s] + np.arange(self.rows[s])[:, None]
        j = np.arange(self.past[s] + self.rows[s])
        ok = j[None] <= p
        if self.window:
            ok &= (j[None] > p - self.window) | (j[None] < self.sinks)
        used = ok.any(0)
        return j[used], torch.from_numpy(ok[:, used])


def attn_ref(q, k_of, v_of, batch, scale):
    """{"out", "lse"}: (value, bound) in float64.  k_of(s, positions): the cached
    values [positions, kv heads, head_dim], float64, of the type of q."""
    dt, (rows, hq, hd) = q.dtype, q.shape
    u, fl, q = unit(dt), floor_of(dt), q.double().cpu()
    out, e_out = torch.zeros(rows, hq, hd, dtype=torch.float64), torch.zeros(rows, hq, hd, dtype=torch.float64)
    lse, e_lse = torch.full((hq, rows), -np.inf, dtype=torch.float64), torch.zeros(hq, rows, dtype=torch.float64)
    for s in range(len(batch.rows)):
        if not batch.rows[s]:
            continue
        j, seen = batch.seen(s)
        K, V = k_of(s, j), v_of(s, j)
        group = hq // K.shape[1]
        sl = slice(int(batch.row_start[s]), int(batch.row_start[s + 1]))
        n = len(j)
        for h in range(hq):
            kh, vh, Q = K[:, h // group], V[:, h // group], q[sl, h]
            sc = (Q @ kh.T * scale).masked_fill(~seen, -np.inf)
            top = torch.logsumexp(sc, -1)
            P = torch.exp(sc - top[:, None])
            # a score's error: hd terms of its product, its scaling, the exponent's argument
            ds = ((Q.abs() @ kh.abs().T * abs(scale)) * seen).amax(-1) * (hd + 8) * F
            rel = 2 * ds[:, None] + (n + 64) * F
            A = P @ vh.abs()
            out[sl, h] = P @ vh
            e_out[sl, h] = u * (A + out[sl, h].abs()) + A * rel + fl * (1 + n * 256 * vh.abs().amax())
            lse[h, sl] = top
            e_lse[h, sl] = ds + (n + 32) * F + 4 * F * top.abs()
    return {"out": (out, e_out), "lse": (lse, e_lse)}


def logits_ref(logits, tokens, row_len, prompt_len, row_seq, repetition=None, presence=None, frequency=None, bias=None,
               mask=None, mask_row=None):
    """(value, bound) in float64, row by row and list by list."""
    dt = logits.dtype
    y = logits.double().cpu().clone()
    mag = y.abs()
    rows, vocab = y.shape
    for r in range(rows):
        s = int(row_seq[r])
        known = 0 <= s < (len(prompt_len) if prompt_len is not None else 1 << 30)
        if tokens is not None and known:
            n = max(0, min(int(row_len[r]), tokens.shape[1]))
            h = [int(t) for t in tokens[s, :n]]
            made = h[max(0, int(prompt_len[s])):]
            for t in set(t for t in h if 0 <= t < vocab):
                if repetition is not None:
                    f = float(repetition[s])
                    y[r, t] = y[r, t] / f if y[r, t] > 0 else y[r, t] * f
                    mag[r, t] = max(mag[r, t], y[r, t].abs())
                c = made.count(t)
                if c and frequency is not None:
                    y[r, t] -= float(frequency[s]) * c
                    mag[r, t] += abs(float(frequency[s])) * c
                if c and presence is not None:
                    y[r, t] -= float(presence[s])
                    mag[r, t] += abs(float(presence[s]))
        if bias is not None and known:
            last = {}
            for i in range(max(0, int(bias[0][s])), min(int(bias[0][s + 1]), len(bias[1]))):
                last[int(bias[1][i])] = float(bias[2][i])
            for t, b in last.items():
                if 0 <= t < vocab:
                    y[r, t] += b
                    mag[r, t] += abs(b)
        if mask is not None:
            m = int(mask_row[r]) if mask_row is not None else r
            if m >= len(mask):
                y[r] = -np.inf
            elif m >= 0:
                for t in range(vocab):
                    if not int(mask[m, t // 32]) >> (t % 32) & 1:
                        y[r, t] = -np.inf
    # five float32 operations, a rounding to the type
    bound = torch.where(torch.isfinite(y), unit(dt) * y.abs() + 6 * F * (1 + unit(dt)) * mag + floor_of(dt), 0.0)
    return y, bound


def best_of(out):
    """Lowest id of the largest value of each row, NaN passed over, -1 if none is above -inf."""
    x = out.float().cpu().numpy().copy()
    x[np.isnan(x)] = -np.inf
    return [int(np.argmax(r)) if r.max() > -np.inf else -1 for r in x]


__all__ = ["DTYPES", "F", "unit", "Batch", "attn_ref", "logits_ref", "stored", "decoded", "best_of", "grid"]
