"""A sharper bound of float16 attention than serve_common's, which grows with the
number of keys until nothing is outside it."""
from __future__ import annotations

import numpy as np
import torch

import serve_common as S
from train_common import floor_of

attn_ref = S.attn_ref


def sharp_attn_ref(q, k_of, v_of, batch, scale):
    """serve_common.attn_ref with what subnormal probabilities lose counted by the
    formula.  A probability is exp(s - m), rounded to half a subnormal step, f =
    2^-25, where it is small; m is a running maximum, so never above the largest
    score M, and a later m scales what was lost down.  The output is divided by
    sum exp(s - m) >= sum exp(s - M), so that all of it is at most
    f sum |v| / sum exp(s - M) over the keys that the row sees."""
    ref = attn_ref(q, k_of, v_of, batch, scale)
    fl = floor_of(q.dtype)
    if not fl:
        return ref
    bound, x = ref["out"][1], q.double().cpu()
    for s in range(len(batch.rows)):
        if not batch.rows[s]:
            continue
        j, seen = batch.seen(s)
        K, V = k_of(s, j), v_of(s, j)
        sl = slice(int(batch.row_start[s]), int(batch.row_start[s + 1]))
        for h in range(q.shape[1]):
            k, v = K[:, h // (q.shape[1] // K.shape[1])], V[:, h // (q.shape[1] // K.shape[1])].abs()
            sc = (x[sl, h] @ k.T * scale).masked_fill(~seen, -np.inf)
            share = torch.exp(sc - sc.amax(-1, keepdim=True)).sum(-1)
            bound[sl, h] += fl * (seen.double() @ v / share[:, None] - len(j) * 256 * v.amax())
    return ref
