"""Mask-token training operators on the CPU: refusals of the C entry points and
the binding (nothing is dereferenced, no device work), and the float64 forms
that the GPU tests compare with: against the oracle's context rule, torch's own
cross entropy, and differences."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import train_common as T
from oracle import cod

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2504_18583_amd", "libpard.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libpard.so not built")
P = 4096                                            # never dereferenced


@pytest.fixture(scope="module")
def b():
    from paper_2504_18583_amd import binding
    return binding


def _rope_args(b, **kw):
    base = dict(rows=4, n_q=2, n_k=1, head_dim=64, dtype=b.PARD_BF16, rot_dim=64, layout=b.PARD_ROPE_HALF, n_pos=16,
                eps=1e-6, positions=P, table=P, q_gain=None, k_gain=None)
    return b.pard_rope_args(**(base | kw))


@needs_lib
@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), "ARG"), (dict(n_q=0), "ARG"), (dict(n_k=-1), "ARG"), (dict(head_dim=1), "ARG"),
    (dict(head_dim=1026, rot_dim=64), "ARG"), (dict(rot_dim=66), "ARG"), (dict(rot_dim=63), "ARG"), (dict(rot_dim=0), "ARG"),
    (dict(n_pos=0), "ARG"), (dict(n_pos=(1 << 24) + 1), "ARG"), (dict(layout=2), "ARG"), (dict(eps=-1.0), "ARG"),
    (dict(eps=float("inf")), "ARG"), (dict(positions=None), "ARG"), (dict(table=None), "ARG"), (dict(table=P + 4), "ARG"),
    (dict(q_gain=P), "ARG"), (dict(k_gain=P), "ARG"), (dict(dtype=3), "UNSUPPORTED"), (dict(dtype=-1), "UNSUPPORTED"),
    (dict(rows=1 << 31), "UNSUPPORTED")])
def test_qk_rope_refuses(b, kw, status):
    h = b.pard_heads(P, 1 << 20, 64)
    want = getattr(b, "PARD_ERR_" + status)
    a = _rope_args(b, **kw)
    assert b.lib.pard_qk_rope(a, h, h, h, h, None) == want
    assert b.lib.pard_qk_rope_grad(a, h, h, h, h, h, h, P, P, P, 1 << 30, None) == want
    assert b.lib.pard_qk_rope_workspace_bytes(a) == 0


@needs_lib
def test_qk_rope_refuses_tensors(b):
    ok, a = b.pard_heads(P, 128, 64), _rope_args(b)
    call = lambda q, k, qo, ko: b.lib.pard_qk_rope(a, q, k, qo, ko, None)  # noqa: E731
    assert b.lib.pard_qk_rope(None, ok, ok, ok, ok, None) == b.PARD_ERR_ARG
    for bad in (None, b.pard_heads(None, 128, 64), b.pard_heads(P, -128, 64), b.pard_heads(P, 128, -1)):
        assert call(bad, ok, ok, ok) == call(ok, bad, ok, ok) == call(ok, ok, bad, ok) == call(ok, ok, ok, bad) == b.PARD_ERR_ARG
    # outputs whose heads overlap: rows too close, heads too close, neither order
    for bad in (b.pard_heads(P, 127, 64), b.pard_heads(P, 128, 63), b.pard_heads(P, 64, 64), b.pard_heads(P, 0, 64)):
        assert call(ok, ok, bad, ok) == b.PARD_ERR_ARG
    # gradients with gains: inputs, gain gradients, workspace
    g = _rope_args(b, q_gain=P, k_gain=P)
    n = b.lib.pard_qk_rope_workspace_bytes(g)
    assert n > 0 and b.lib.pard_qk_rope_workspace_bytes(a) == 0
    grad = lambda q=ok, k=ok, dg=P, dk=P, ws=P, nb=n: b.lib.pard_qk_rope_grad(g, ok, ok, q, k, ok, ok, dg, dk, ws, nb, None)  # noqa: E731
    assert grad(q=None) == grad(k=None) == grad(dg=None) == grad(dk=None) == grad(ws=None) == grad(ws=P + 128) == b.PARD_ERR_ARG
    assert grad(nb=n - 1) == b.PARD_ERR_NOMEM
    # nothing to do: accepted without tensors' data
    none = b.pard_heads(None, 0, 0)
    assert b.lib.pard_qk_rope(_rope_args(b, rows=0, positions=None, table=None), none, none, none, none, None) == b.PARD_OK


@needs_lib
def test_rope_table_refuses(b):
    def spec(**kw):
        base = dict(rot_dim=64, scaling=b.PARD_ROPE_YARN, theta=1e4, factor=4.0, low=1.0, high=32.0, original_max_pos=4096)
        return b.pard_rope_spec(**(base | kw))
    size = lambda s, n=8: b.lib.pard_rope_table_bytes(s, n)  # noqa: E731
    assert size(spec()) == 8 * 64 * 4 and size(spec(scaling=b.PARD_ROPE_PLAIN, factor=0.0)) == 2048
    for bad in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=1026), dict(scaling=4), dict(scaling=-1), dict(theta=1.0),
                dict(theta=float("inf")), dict(factor=0.5), dict(factor=float("nan")), dict(low=0.0), dict(high=1.0),
                dict(original_max_pos=0)):
        assert size(spec(**bad)) == 0, bad
        assert b.lib.pard_rope_table(spec(**bad), 8, P, None) == b.PARD_ERR_ARG
    assert size(spec(), 0) == 0 and size(spec(), (1 << 24) + 1) == 0
    assert b.lib.pard_rope_table(spec(), 8, None, None) == b.PARD_ERR_ARG
    assert b.lib.pard_rope_table(spec(), 8, P + 8, None) == b.PARD_ERR_ARG


@needs_lib
def test_cod_plan_refuses(b):
    def build(offs, n=None, data=P, n_bytes=1 << 40, sec=P, col=P, lens=P, plan=True):
        o = (C.c_int64 * len(offs))(*offs)
        out = b.pard_cod_plan()
        return b.lib.pard_cod_plan_build(sec, col, C.cast(o, C.POINTER(C.c_int64)), lens, len(offs) - 1 if n is None else n, data,
                                         n_bytes, None, out if plan else None)
    assert build([0, 10], n=0) == build([0, 10, 9]) == build([-1, 10]) == b.PARD_ERR_ARG
    assert build([0, 10], data=None) == build([0, 10], data=P + 128) == build([0, 10], sec=None) == b.PARD_ERR_ARG
    assert build([0, 10], col=None) == build([0, 10], lens=None) == build([0, 10], plan=False) == b.PARD_ERR_ARG
    assert build([0, 64 * 8192 + 1]) == build([(1 << 31) - 5, 1 << 31]) == b.PARD_ERR_UNSUPPORTED
    need = b.lib.pard_cod_plan_bytes(10, 1)
    assert build([0, 10], n_bytes=need - 1) == b.PARD_ERR_NOMEM
    assert need > 0 and b.lib.pard_cod_plan_bytes(-1, 1) == 0 and b.lib.pard_cod_plan_bytes(10, 0) == 0
    assert b.lib.pard_cod_plan_bytes(1 << 31, 1) == 0


@needs_lib
def test_cod_attn_refuses(b):
    plan = b.pard_cod_plan(100, 1, 1, P)
    def args(**kw):
        base = dict(plan=C.pointer(plan), n_heads=4, n_kv_heads=2, head_dim=64, dtype=b.PARD_BF16, scale=0.125)
        return b.pard_cod_attn_args(**(base | kw))
    h = b.pard_heads(P, 256, 64)
    unbuilt = b.pard_cod_plan()
    cases = [(dict(plan=None), "ARG"), (dict(plan=C.pointer(unbuilt)), "ARG"), (dict(n_heads=0), "ARG"), (dict(n_kv_heads=0), "ARG"),
             (dict(n_kv_heads=3), "ARG"), (dict(scale=float("nan")), "ARG"), (dict(head_dim=96), "UNSUPPORTED"),
             (dict(dtype=b.PARD_F32), "UNSUPPORTED"), (dict(dtype=7), "UNSUPPORTED"), (dict(n_heads=65536, n_kv_heads=1), "UNSUPPORTED")]
    for kw, status in cases:
        a, want = args(**kw), getattr(b, "PARD_ERR_" + status)
        assert b.lib.pard_cod_attn(a, h, h, h, h, P, None) == want, kw
        assert b.lib.pard_cod_attn_grad(a, h, h, h, h, h, P, h, h, h, P, 1 << 40, None) == want, kw
        assert b.lib.pard_cod_attn_workspace_bytes(a) == 0
    a = args()
    n = b.lib.pard_cod_attn_workspace_bytes(a)
    assert n >= 4 * 100 * 4
    bad = [None, b.pard_heads(None, 256, 64), b.pard_heads(P + 8, 256, 64), b.pard_heads(P, 260, 64), b.pard_heads(P, 256, 68),
           b.pard_heads(P, -256, 64)]
    for t in bad:
        for i in range(4):
            ts = [h] * 4
            ts[i] = t
            assert b.lib.pard_cod_attn(a, *ts, P, None) == b.PARD_ERR_ARG
        for i in range(8):
            ts = [h] * 8
            ts[i] = t
            assert b.lib.pard_cod_attn_grad(a, *ts[:5], P, *ts[5:], P, n, None) == b.PARD_ERR_ARG
    assert b.lib.pard_cod_attn(a, h, h, h, b.pard_heads(P, 64, 64), P, None) == b.PARD_ERR_ARG       # rows of out overlap
    grad = lambda lse=P, ws=P, nb=n: b.lib.pard_cod_attn_grad(a, h, h, h, h, h, lse, h, h, h, ws, nb, None)  # noqa: E731
    assert grad(lse=None) == grad(ws=None) == grad(ws=P + 64) == b.PARD_ERR_ARG and grad(nb=n - 1) == b.PARD_ERR_NOMEM


@needs_lib
def test_cod_loss_refuses(b):
    def args(**kw):
        base = dict(rows=4, vocab=10, dtype=b.PARD_F32, n_sections=2, grad_scale=1.0, logits=P, logits_stride=10, labels=P,
                    section=P, weights=None, d_logits=P, d_stride=10, loss=P, row_loss=None)
        return b.pard_cod_loss_args(**(base | kw))
    call = lambda ws=P, nb=1 << 30, **kw: b.lib.pard_cod_loss(args(**kw), ws, nb, None)  # noqa: E731
    w = (C.c_float * 2)(1.0, float("inf"))
    for kw in (dict(rows=-1), dict(vocab=0), dict(n_sections=0), dict(n_sections=65), dict(grad_scale=float("nan")), dict(logits=None),
               dict(labels=None), dict(section=None), dict(loss=None), dict(logits_stride=9), dict(d_stride=9), dict(weights=w),
               dict(logits=P + 2), dict(d_logits=P + 2), dict(ws=None), dict(ws=P + 8)):
        assert call(**kw) == b.PARD_ERR_ARG, kw
    assert call(dtype=5) == call(rows=1 << 31) == b.PARD_ERR_UNSUPPORTED
    n = b.lib.pard_cod_loss_workspace_bytes(args())
    assert n > 0 and call(nb=n - 1) == b.PARD_ERR_NOMEM
    assert b.lib.pard_cod_loss_workspace_bytes(args(rows=-1)) == 0


@needs_lib
def test_outputs_on_other_tensors_are_refused(b):
    """An output that starts where another tensor does: refused, but for the
    rotation and the loss in place with the same strides."""
    h = lambda i, rs=256, hs=64: b.pard_heads(P * (i + 1), rs, hs)  # noqa: E731
    a, n = _rope_args(b), 1 << 30
    rope = lambda q, k, qo, ko: b.lib.pard_qk_rope(a, q, k, qo, ko, None)  # noqa: E731
    assert rope(h(0), h(1), h(0, 512), h(2)) == rope(h(0), h(1), h(0, 256, 128), h(2)) == rope(h(0), h(1), h(1), h(2)) == b.PARD_ERR_ARG
    assert rope(h(0), h(1), h(2), h(0)) == rope(h(0), h(1), h(2), h(2)) == rope(h(0), h(1), h(2), h(1, 512)) == b.PARD_ERR_ARG
    g = _rope_args(b, q_gain=P, k_gain=P)
    grad = lambda qd, kd, qo, ko: b.lib.pard_qk_rope_grad(g, qd, kd, h(0), h(1), qo, ko, P, P, P, n, None)  # noqa: E731
    for t in ((h(2), h(3), h(2, 512), h(4)), (h(2), h(3), h(0), h(4)), (h(2), h(3), h(4), h(1)), (h(2), h(3), h(3), h(4)),
              (h(2), h(3), h(4), h(2)), (h(2), h(3), h(4), h(4)), (h(2), h(3), h(1), h(4)), (h(2), h(3), h(4), h(0))):
        assert grad(*t) == b.PARD_ERR_ARG
    plan = b.pard_cod_plan(100, 1, 1, P)
    at = b.pard_cod_attn_args(plan=C.pointer(plan), n_heads=4, n_kv_heads=2, head_dim=64, dtype=b.PARD_BF16, scale=0.125)
    for i in range(3):
        assert b.lib.pard_cod_attn(at, h(0), h(1), h(2), h(i), P, None) == b.PARD_ERR_ARG
    for o in range(3):                               # dq, dk, dv at one of the inputs, or at each other
        for i in range(8):
            if i != 5 + o:
                outs = [h(5), h(6), h(7)]
                outs[o] = h(i)
                assert b.lib.pard_cod_attn_grad(at, h(0), h(1), h(2), h(3), h(4), P, *outs, P, 1 << 40, None) == b.PARD_ERR_ARG
    loss = b.pard_cod_loss_args(rows=4, vocab=10, dtype=b.PARD_F32, n_sections=1, grad_scale=1.0, logits=P, logits_stride=10, labels=P,
                                section=None, weights=None, d_logits=P, d_stride=12, loss=P, row_loss=None)
    assert b.lib.pard_cod_loss(loss, P, 1 << 30, None) == b.PARD_ERR_ARG


@needs_lib
def test_sizes_past_a_launch_are_refused(b):
    def attn(n_tiles, nq, nk):
        plan = b.pard_cod_plan(100, 1, n_tiles, P)
        a = b.pard_cod_attn_args(plan=C.pointer(plan), n_heads=nq, n_kv_heads=nk, head_dim=64, dtype=b.PARD_BF16, scale=0.125)
        return b.lib.pard_cod_attn(a, *[b.pard_heads(P, 256, 64)] * 4, P, None), b.lib.pard_cod_attn_workspace_bytes(a)
    assert attn(1 << 21, 8, 1) == attn(1 << 19, 8, 8) == (b.PARD_ERR_UNSUPPORTED, 0)
    assert attn(1, 1025, 1) == (b.PARD_ERR_UNSUPPORTED, 0)
    assert attn((1 << 21) - 1, 8, 1)[1] > 0
    offs = (C.c_int64 * ((1 << 22) + 1))()
    got = b.lib.pard_cod_plan_build(P, P, C.cast(offs, C.POINTER(C.c_int64)), P, 1 << 22, P, 1 << 40, None, b.pard_cod_plan())
    assert got == b.PARD_ERR_UNSUPPORTED
    h = lambda rs: b.pard_heads(P, rs, 64)  # noqa: E731
    plan = b.pard_cod_plan(100, 1, 1, P)
    a = b.pard_cod_attn_args(plan=C.pointer(plan), n_heads=4, n_kv_heads=2, head_dim=64, dtype=b.PARD_BF16, scale=0.125)
    assert b.lib.pard_cod_attn(a, h(1 << 31), h(256), h(256), h(256), P, None) == b.PARD_ERR_ARG
    assert b.lib.pard_cod_attn(a, b.pard_heads(P, 256, 1 << 31), h(256), h(256), h(256), P, None) == b.PARD_ERR_ARG
    for bad in (float("inf"), float("-inf"), float("nan")):
        a.scale = bad
        assert b.lib.pard_cod_attn(a, h(256), h(256), h(256), h(256), P, None) == b.PARD_ERR_ARG


@needs_lib
def test_binding_refuses_what_no_pointer_shows(b):
    """Tensors that the binding turns away before it calls the library (host
    tensors here, as any tensor that is not on a GPU)."""
    q, t = torch.zeros(4, 2, 64), torch.zeros(16, 32, 2)
    with pytest.raises(b.PardError, match="device tensor"):
        b.qk_rope(q, None, torch.zeros(4, dtype=torch.int32), t)
    with pytest.raises(b.PardError, match="ascending"):
        b.cod_plan(torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), [0, 3, 2], torch.zeros(2, dtype=torch.int32))
    with pytest.raises(b.PardError, match="section"):
        b.cod_plan(torch.zeros(4), torch.zeros(4, dtype=torch.int32), [0, 4], torch.zeros(1, dtype=torch.int32))
    with pytest.raises(b.PardError, match="contiguous rows"):
        b.cod_loss(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), None, 1)
    with pytest.raises(b.PardError, match="scaling"):
        b.rope_table(8, 64, 1e4, scaling="ntk", device="cpu")


# ---- the float64 forms --------------------------------------------------------

def test_seen_mask_is_the_oracles():
    for n, k, r in ((9, 4, 0.7), (23, 8, 0.7), (12, 1, 0.7), (30, 12, 1.0)):
        s = cod.cod_process(list(range(n + 1)), k, r, 0.2, 0, 5, 2)
        assert np.array_equal(T.seen_mask(s.section, s.column).numpy(), cod.attention_mask(s))


def test_attention_form_against_differences():
    torch.manual_seed(0)
    section, column, offs, lens, rows = T.pack([7, 0, 4], 3, slack=2, lead=1, trail=1)
    q, k, v, g = (torch.randn(rows, h, 8, dtype=torch.float64) for h in (4, 2, 2, 4))
    T_unit, T.unit = T.unit, lambda dt: 0.0
    try:
        ref = T.attn_ref(q, k, v, section, column, offs, lens, 0.3, g)
        inside = torch.zeros(rows, dtype=torch.bool)
        for o, n in zip(offs, lens):
            inside[o:o + n] = True
        value = lambda: (T.attn_ref(q, k, v, section, column, offs, lens, 0.3)["out"][0] * g)[inside].sum()  # noqa: E731
        eps = 1e-5
        for t, name in ((q, "dq"), (k, "dk"), (v, "dv")):
            for at in [(int(offs[0]), 1, 3), (int(offs[0]) + 5, 0, 0), (int(offs[2]) + 2, 1, 7), (0, 0, 0), (rows - 1, 1, 1)]:
                x = float(t[at])
                t[at] = x + eps
                up = value()
                t[at] = x - eps
                down = value()
                t[at] = x
                assert abs((up - down) / (2 * eps) - ref[name][0][at]) < 1e-8, (name, at)
    finally:
        T.unit = T_unit


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_form_against_autograd(layout, norm):
    torch.manual_seed(1)
    x = torch.randn(5, 3, 16, dtype=torch.float64, requires_grad=True)
    gain = (1 + 0.1 * torch.randn(16, dtype=torch.float64)).requires_grad_(norm) if norm else None
    table = torch.randn(9, 5, 2, dtype=torch.float64)              # (any table: 10 of 16 dims turned)
    pos, dy = torch.tensor([3, 0, 8, 3, 1]), torch.randn(5, 3, 16, dtype=torch.float64)
    n = x if gain is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-3) * gain
    cs = table[pos][:, None]
    y = T.turn(n, cs[..., 0], cs[..., 1], layout)
    want = torch.autograd.grad(y, (x, gain) if norm else (x,), dy)
    dx, _, dg, _ = T.rope_grad_ref(dy, x.detach(), pos, table, layout, None if gain is None else gain.detach(), 1e-3)
    assert torch.allclose(dx, want[0], atol=1e-12)
    if norm:
        assert torch.allclose(dg, want[1], atol=1e-12)


@pytest.mark.parametrize("weights", [None, [0.5, 2.0, 0.25]])
def test_loss_form_against_torch(weights):
    torch.manual_seed(2)
    x = torch.randn(20, 11, dtype=torch.float64, requires_grad=True)
    labels = torch.randint(-1, 11, (20,))
    section = torch.randint(1, 4, (20,))
    ce = torch.nn.functional.cross_entropy(x, labels.clamp(min=0), reduction="none") * (labels >= 0)
    parts = [ce[(section == k) & (labels >= 0)].mean() for k in (1, 2, 3)]
    loss = ce.sum() / (labels >= 0).sum() if weights is None else sum(w * p for w, p in zip(weights, parts))
    d, = torch.autograd.grad(3.0 * loss, x)
    got = T.loss_ref(x.detach(), labels, section, 3, weights, 3.0)
    assert abs(got[0] - loss.detach()) < 1e-12 and torch.allclose(got[1], torch.stack(parts).detach()) and torch.allclose(got[3], d)
