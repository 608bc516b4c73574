"""Serving operators on the CPU: refusals of the C entry points and the binding
(nothing is dereferenced, no device work), and the float64 forms that the GPU
tests compare with, against torch's own."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import serve_common as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2504_18583_amd", "libpard.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libpard.so not built")
P = 4096                                            # never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2504_18583_amd import binding
    return binding


def _cache(b, **kw):
    base = dict(n_pages=8, page_size=16, n_kv_heads=2, head_dim=64, dtype=b.PARD_E4M3, k=P, v=2 * P, k_scale=3 * P, v_scale=4 * P)
    return b.pard_kv_cache(**(base | kw))


def _batch(b, **kw):
    base = dict(rows=4, n_seqs=2, max_pages=3, max_seq_rows=0, page_table=P, row_start=P, kv_len=P)
    return b.pard_kv_batch(**(base | kw))


CACHES = [(dict(n_pages=0), "ARG"), (dict(page_size=8), "ARG"), (dict(page_size=24), "ARG"), (dict(page_size=8192), "ARG"),
          (dict(n_kv_heads=0), "ARG"), (dict(k=None), "ARG"), (dict(v=None), "ARG"), (dict(k=P + 8), "ARG"), (dict(v=P + 4), "ARG"),
          (dict(k_scale=None), "ARG"), (dict(v_scale=None), "ARG"), (dict(k_scale=P + 2), "ARG"), (dict(v_scale=P + 1), "ARG"),
          (dict(dtype=0), "UNSUPPORTED"), (dict(dtype=5), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"),
          (dict(n_kv_heads=65536), "UNSUPPORTED")]
BATCHES = [(dict(rows=-1), "ARG"), (dict(n_seqs=0), "ARG"), (dict(max_pages=0), "ARG"), (dict(max_seq_rows=-1), "ARG"),
           (dict(page_table=None), "ARG"), (dict(row_start=None), "ARG"), (dict(kv_len=None), "ARG"), (dict(rows=1 << 30), "UNSUPPORTED"),
           (dict(n_seqs=(1 << 20) + 1), "UNSUPPORTED"), (dict(max_pages=(1 << 26) + 1), "UNSUPPORTED")]


@needs_lib
def test_caches_and_batches_are_checked(b):
    h, o = b.pard_heads(8 * P, 1 << 20, 64), b.pard_heads(9 * P, 1 << 20, 64)
    cases = [(_cache(b, **kw), _batch(b), s) for kw, s in CACHES] + [(_cache(b), _batch(b, **kw), s) for kw, s in BATCHES]
    for cache, batch, status in cases + [(None, _batch(b), "ARG"), (_cache(b), None, "ARG")]:
        want = getattr(b, "PARD_ERR_" + status)
        assert b.lib.pard_kv_write(cache, batch, b.PARD_BF16, h, o, None) == want
        assert b.lib.pard_kv_read(cache, batch, b.PARD_BF16, h, o, None) == want
        pc, pb = C.pointer(cache) if cache else None, C.pointer(batch) if batch else None
        a = b.pard_kv_attn_args(pc, pb, 4, b.PARD_BF16, 0, 0, 0.125)
        assert b.lib.pard_kv_attn(a, h, o, P, P, 1 << 40, None) == want
        assert b.lib.pard_kv_attn_workspace_bytes(a) == 0


@needs_lib
def test_rows_are_checked(b):
    cache, batch = _cache(b), _batch(b)
    ok, other = b.pard_heads(8 * P, 128, 64), b.pard_heads(9 * P, 128, 64)
    for call, outputs in ((b.lib.pard_kv_write, False), (b.lib.pard_kv_read, True)):
        f = lambda k, v, dt=b.PARD_BF16: call(cache, batch, dt, k, v, None)  # noqa: E731
        assert f(ok, other, 3) == f(ok, other, -1) == b.PARD_ERR_UNSUPPORTED
        for bad in (None, b.pard_heads(None, 128, 64), b.pard_heads(8 * P, -1, 64), b.pard_heads(8 * P, 128, -1), b.pard_heads(8 * P + 1, 128, 64)):
            assert f(bad, other) == f(ok, bad) == b.PARD_ERR_ARG
        assert f(b.pard_heads(8 * P + 2, 128, 64), other, b.PARD_F32) == b.PARD_ERR_ARG
        if outputs:                                  # heads that overlap, one tensor for both, the cache itself
            assert f(b.pard_heads(8 * P, 127, 64), other) == f(ok, b.pard_heads(9 * P, 128, 63)) == f(ok, ok) == b.PARD_ERR_ARG
            assert f(b.pard_heads(P, 128, 64), other) == f(ok, b.pard_heads(2 * P, 128, 64)) == b.PARD_ERR_ARG
        none = b.pard_heads(None, 0, 0)
        assert call(cache, _batch(b, rows=0), b.PARD_BF16, none, none, None) == b.PARD_OK


@needs_lib
def test_kv_attn_refuses(b):
    cache, batch = _cache(b), _batch(b)
    def args(**kw):
        base = dict(cache=C.pointer(cache), batch=C.pointer(batch), n_heads=4, dtype=b.PARD_BF16, window=0, sinks=0, scale=0.125)
        return b.pard_kv_attn_args(**(base | kw))
    q, o = b.pard_heads(8 * P, 256, 64), b.pard_heads(9 * P, 256, 64)
    n = b.lib.pard_kv_attn_workspace_bytes(args())
    assert n > 0
    call = lambda a=None, q=q, o=o, ws=P, nb=n: b.lib.pard_kv_attn(a or args(), q, o, P, ws, nb, None)  # noqa: E731
    assert b.lib.pard_kv_attn(None, q, o, P, P, n, None) == b.PARD_ERR_ARG
    for kw in (dict(n_heads=0), dict(n_heads=3), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(sinks=-1)):
        assert call(args(**kw), nb=1 << 40) == b.PARD_ERR_ARG and b.lib.pard_kv_attn_workspace_bytes(args(**kw)) == 0
    same = _cache(b, dtype=b.PARD_F16, k_scale=None, v_scale=None)
    large = _batch(b, rows=1 << 29)
    for kw in (dict(dtype=b.PARD_F32), dict(dtype=3), dict(cache=C.pointer(same)), dict(n_heads=2050), dict(batch=C.pointer(large), n_heads=8)):
        assert call(args(**kw), nb=1 << 50) == b.PARD_ERR_UNSUPPORTED and b.lib.pard_kv_attn_workspace_bytes(args(**kw)) == 0
    for bad in (None, b.pard_heads(None, 256, 64), b.pard_heads(8 * P + 8, 256, 64), b.pard_heads(8 * P, 260, 64), b.pard_heads(8 * P, 256, 68),
                b.pard_heads(8 * P, -256, 64), b.pard_heads(8 * P, 1 << 31, 64)):
        assert call(q=bad) == call(o=bad) == b.PARD_ERR_ARG
    assert call(o=b.pard_heads(9 * P, 64, 64)) == call(o=q) == call(o=b.pard_heads(P, 256, 64)) == b.PARD_ERR_ARG
    assert call(ws=None) == call(ws=P + 128) == b.PARD_ERR_ARG and call(nb=n - 1) == b.PARD_ERR_NOMEM


@needs_lib
def test_logits_adjust_refuses(b):
    def args(**kw):
        base = dict(rows=4, vocab=70, dtype=b.PARD_F32, n_seqs=4, logits=P, logits_stride=70, out=2 * P, out_stride=70, tokens=P, tokens_stride=9,
                    row_len=P, best=P)
        return b.pard_logits_args(**(base | kw))
    call = lambda ws=P, nb=1 << 30, **kw: b.lib.pard_logits_adjust(args(**kw), ws, nb, None)  # noqa: E731
    for kw in (dict(rows=-1), dict(vocab=0), dict(n_seqs=0), dict(logits=None), dict(out=None), dict(logits=P + 2), dict(out=P + 1),
               dict(logits_stride=69), dict(out_stride=69), dict(logits_stride=-70), dict(out=P, out_stride=72), dict(n_seqs=3),
               dict(row_len=None), dict(tokens_stride=-1), dict(tokens=None, repetition=P), dict(tokens=None, presence=P),
               dict(tokens=None, frequency=P), dict(bias_start=P, n_bias=-1), dict(bias_start=P, n_bias=1, bias_ids=P),
               dict(bias_start=P, n_bias=1, bias_values=P), dict(mask=P, n_masks=-1, mask_stride=3), dict(mask=P, n_masks=4, mask_stride=2),
               dict(ws=None), dict(ws=P + 8)):
        assert call(**kw) == b.PARD_ERR_ARG, kw
    assert call(dtype=3) == call(rows=1 << 30, n_seqs=1 << 30) == call(vocab=(1 << 28) + 1) == b.PARD_ERR_UNSUPPORTED
    n = b.lib.pard_logits_workspace_bytes(args())
    assert n > 0 and call(nb=n - 1) == b.PARD_ERR_NOMEM
    assert b.lib.pard_logits_workspace_bytes(args(best=None)) == b.lib.pard_logits_workspace_bytes(args(rows=-1)) == 0
    assert b.lib.pard_logits_adjust(None, P, n, None) == b.PARD_ERR_ARG
    assert call(rows=0, logits=None, out=None) == b.PARD_OK


@needs_lib
def test_binding_refuses_what_no_pointer_shows(b):
    z, i = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(b.PardError, match="device tensor"):
        b.KVCache(z, z)
    with pytest.raises(b.PardError, match="device tensor"):
        b.KVBatch(i, i[0], i[0])
    with pytest.raises(b.PardError, match="device tensor"):
        b.logits_adjust(torch.zeros(2, 8))
    for f in (lambda x: b.kv_write(x, x, None, None), lambda x: b.kv_attn(x, None, None), lambda x: b.logits_adjust(x[0])):
        with pytest.raises(b.PardError, match="no gradient") as e:
            f(torch.zeros(2, 2, 64, requires_grad=True))
        assert e.value.status == b.PARD_ERR_ARG
    with pytest.raises(b.PardError, match="head_dim"):
        b.kv_cache(2, 16, 1, 50, "e4m3", device="cpu")


# --------------------------------------------------------------------------
# the float64 forms
# --------------------------------------------------------------------------

def test_grids_are_the_formats():
    """torch's own e4m3 for all its codes; e2m1's eight values."""
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double()
    got = S.decoded(codes.view(8, 32), torch.full((8, 1), 127, dtype=torch.uint8), "e4m3").flatten()
    assert torch.equal(got[~want.isnan()], want[~want.isnan()]) and torch.equal(got.isnan(), want.isnan())
    assert S.grid("e2m1").tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]


def test_stored_blocks():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(64, 32, generator=g) * torch.exp2(torch.randint(-60, 60, (64, 1), generator=g).float())
    for cache, top in (("e4m3", 448.0), ("e2m1", 6.0)):
        y, big = S.stored(x, cache), x.abs().amax(-1, keepdim=True).double()
        scale = torch.exp2(torch.ceil(torch.log2(big / top)))
        if cache == "e4m3":                          # torch's rounding to the type, under the scale
            assert torch.equal(y, (x / scale).to(torch.float8_e4m3fn).double() * scale)
        step = scale * (32 if cache == "e4m3" else 2)
        assert bool(((y - x).abs() <= step / 2).all()) and bool((y.abs() <= top * scale).all())
    edge = torch.zeros(4, 32)
    edge[0, 0], edge[1, 0], edge[2, 3], edge[3, 31] = 448.0, 448.5, float("inf"), float("nan")
    y = S.stored(edge, "e4m3")
    assert y[0, 0] == 448 and y[1, 0] == 448 and y[2:].isnan().all() and (y[:2, 1:] == 0).all()
    assert S.stored(torch.tensor([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4]), "e2m1")[0, :8].tolist() == [0, 1, 1, 2, 2, 4, 4, 6]


@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 0), (5, 2), (1, 40), (100, 1)])
def test_attention_form_matches_torch(window, sinks):
    g = torch.Generator().manual_seed(2)
    batch = S.Batch([1, 7, 0, 12], [0, 20, 9, 3], 16, window, sinks)
    K, V = torch.randn(4, 64, 2, 64, generator=g, dtype=torch.float64), torch.randn(4, 64, 2, 64, generator=g, dtype=torch.float64)
    q = torch.randn(batch.n, 4, 64, generator=g)
    got = S.attn_ref(q, lambda s, j: K[s, j], lambda s, j: V[s, j], batch, 0.3)
    for s, (m, p) in enumerate(zip(batch.rows, batch.past)):
        sl, n = slice(int(batch.row_start[s]), int(batch.row_start[s + 1])), m + p
        i, j = torch.arange(p, n)[:, None], torch.arange(n)[None]
        mask = (j <= i) & ((j > i - window) | (j < sinks) if window else True)
        want = torch.nn.functional.scaled_dot_product_attention(
            q[sl].double().transpose(0, 1), K[s, :n].repeat_interleave(2, 1).transpose(0, 1), V[s, :n].repeat_interleave(2, 1).transpose(0, 1),
            attn_mask=mask, scale=0.3)
        assert torch.allclose(got["out"][0][sl], want.transpose(0, 1), rtol=0, atol=1e-12)


def test_logits_form_on_a_worked_row():
    y, _ = S.logits_ref(torch.tensor([[2.0, -2.0, 1.0, 4.0]]), torch.tensor([[0, 1, 0, 0, 9]]), [5], [1], [0], torch.tensor([2.0]),
                        torch.tensor([0.25]), torch.tensor([0.5]), (torch.tensor([0, 2]), torch.tensor([2, 2]), torch.tensor([7.0, 8.0])),
                        np.array([[0b0111]]))
    # id 0: 2 / 2 - 2 * 0.5 - 0.25; id 1: -2 * 2 - 0.5 - 0.25; id 2: the later bias; id 3: not allowed
    assert y.tolist() == [[-0.25, -4.75, 9.0, -np.inf]] and S.best_of(y) == [2]
    assert S.best_of(torch.tensor([[float("nan"), 1.0, 1.0], [-np.inf] * 3, [-0.0, 0.0, -1.0]])) == [1, -1, 0]
