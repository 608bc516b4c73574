"""GPU checks of the mask-token training operators (rotary positions, attention
over packed COD rows, the loss) against plain float64 forms, element by element
within derived bounds (train_common)."""
import numpy as np
import pytest
import torch

import train_common as T
from gpu_common import require_gpu, say

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def B():
    require_gpu()
    from paper_2504_18583_amd import binding
    return binding


def _randn(gen, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# --------------------------------------------------------------------------
# rotary positions
# --------------------------------------------------------------------------

# rows, query heads, key heads, head_dim, turned dims
ROPE_SHAPES = [(1, 1, 1, 64, 64), (3, 2, 1, 64, 32), (67, 14, 2, 64, 64), (40, 32, 8, 128, 128), (33, 5, 1, 80, 80), (9, 3, 3, 96, 48),
               (7, 4, 2, 256, 128), (5, 2, 2, 6, 4), (4, 3, 1, 34, 34), (300, 1, 1, 2, 2), (6, 2, 1, 1024, 1024), (11, 2, 0, 64, 64),
               (129, 7, 3, 112, 16), (2, 1, 1, 512, 512), (2, 1, 1, 528, 528),
               (41, 5, 1, 80, 40), (13, 3, 2, 24, 8), (70, 8, 8, 40, 40), (5, 2, 1, 264, 136), (3, 2, 2, 504, 8), (500, 3, 1, 72, 24),
               (2500, 2, 1, 64, 64), (3000, 1, 1, 8, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", ROPE_SHAPES, ids=str)
def test_rope_forward_and_gradient(B, shape, layout, dtype):
    rows, hq, hk, hd, rot = shape
    g, dt = _gen(rows + hd), T.DTYPES[dtype]
    say(f"[gpu] rope {shape} {layout} {dtype}")
    n_pos = 50
    table = B.rope_table(n_pos, rot, 1e4)
    pos = torch.randint(0, n_pos, (rows,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = n_pos - 1
    # one projection's output: strided heads
    qkv = _randn(g, rows, (hq + 2 * hk) * hd, dtype=dt)
    q, k = qkv[:, :hq * hd].unflatten(1, (hq, hd)), qkv[:, hq * hd:(hq + hk) * hd].unflatten(1, (hk, hd)) if hk else None
    for norm in (False, True):
        gq = 1 + _randn(g, hd, std=0.2) if norm else None
        gk = 1 + _randn(g, hd, std=0.2) if norm and hk else None
        yq, yk = B.qk_rope(q, k, pos, table, layout, gq, gk, eps=1e-5)
        dq, dk = _randn(g, rows, hq, hd, dtype=dt), _randn(g, rows, hk, hd, dtype=dt) if hk else None
        xq, xk, gdq, gdk = B.qk_rope_grad(dq, dk, pos, table, layout, q, k, gq, gk, eps=1e-5)
        for name, x, y, gain, dy, dx, dg in (("q", q, yq, gq, dq, xq, gdq), ("k", k, yk, gk, dk, xk, gdk)):
            if x is None:
                assert y is None and dx is None and dg is None
                continue
            T.assert_within(y, *T.rope_ref(x, pos, table, layout, gain, 1e-5), f"{name} norm={norm}")
            want, bound, want_g, bound_g = T.rope_grad_ref(dy, x, pos, table, layout, gain, 1e-5)
            T.assert_within(dx, want, bound, f"d{name} norm={norm}")
            if norm:
                T.assert_within(dg, want_g, bound_g, f"d{name} gain")
            else:
                assert dg is None


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("hd", [64, 128])
def test_rope_in_place_head_major_and_odd_strides(B, hd, norm):
    """Outputs that are the inputs, tensors laid out [heads][rows], and rows at
    odd element offsets (which no 16-byte access fits)."""
    g = _gen(3)
    rows, table = 77, B.rope_table(128, hd, 5e5)
    pos = torch.randint(0, 128, (rows,), generator=g, device="cuda", dtype=torch.int32)
    gq, gk = (1 + _randn(g, hd, std=0.1), 1 + _randn(g, hd, std=0.1)) if norm else (None, None)
    q, k = _randn(g, rows, 4, hd, dtype=torch.bfloat16), _randn(g, rows, 2, hd, dtype=torch.bfloat16)
    dy, dyk = _randn(g, rows, 4, hd, dtype=torch.bfloat16), _randn(g, rows, 2, hd, dtype=torch.bfloat16)
    want = B.qk_rope(q, k, pos, table, "half", gq, gk)
    want_d = B.qk_rope_grad(dy, dyk, pos, table, "half", q, k, gq, gk)
    say("[gpu] rope in place")
    a, b = q.clone(), k.clone()
    got = B.qk_rope(a, b, pos, table, "half", gq, gk, q_out=a, k_out=b)
    assert got[0] is a and torch.equal(a, want[0]) and torch.equal(b, want[1])
    a, b = dy.clone(), dyk.clone()
    got = B.qk_rope_grad(a, b, pos, table, "half", q, k, gq, gk, q_dx=a, k_dx=b)
    assert torch.equal(a, want_d[0]) and torch.equal(b, want_d[1])
    if norm:
        assert torch.equal(got[2], want_d[2]) and torch.equal(got[3], want_d[3])

    def place(t, how):
        rows, h, hd = t.shape
        if how == "head-major":
            s = torch.full((h, rows, hd), NAN, device="cuda", dtype=t.dtype).transpose(0, 1)
        else:
            s = torch.full((rows * (h * hd + 3) + 1,), NAN, device="cuda", dtype=t.dtype)[1:].view(rows, -1)[:, :h * hd].unflatten(1, (h, hd))
        return s.copy_(t)
    for how in ("head-major", "odd"):
        say(f"[gpu] rope {how}")
        o, ok = place(torch.zeros_like(q), how), place(torch.zeros_like(k), how)
        B.qk_rope(place(q, how), place(k, how), pos, table, "half", gq, gk, q_out=o, k_out=ok)
        T.assert_within(o, *T.rope_ref(q, pos, table, "half", gq, 1e-6), how)
        T.assert_within(ok, *T.rope_ref(k, pos, table, "half", gk, 1e-6), how)
        got = B.qk_rope_grad(place(dy, how), place(dyk, how), pos, table, "half", place(q, how), place(k, how), gq, gk)
        for i, (d, x, gain) in enumerate(((dy, q, gq), (dyk, k, gk))):
            w, bd, wg, bg = T.rope_grad_ref(d, x, pos, table, "half", gain, 1e-6)
            T.assert_within(got[i], w, bd, how)
            if norm:
                T.assert_within(got[2 + i], wg, bg, how)


def test_rope_positions_outside_the_table_and_no_rows(B):
    table = B.rope_table(8, 64, 1e4)
    q = torch.ones(4, 2, 64, device="cuda")
    pos = torch.tensor([0, 8, -1, 7], dtype=torch.int32, device="cuda")
    y, none = B.qk_rope(q, None, pos, table)
    assert none is None and y[[0, 3]].isfinite().all() and y[[1, 2]].isnan().all()
    g = torch.ones(64, device="cuda")
    d, _, dg, _ = B.qk_rope_grad(q, None, pos, table, q=q, q_gain=g)
    assert d[[0, 3]].isfinite().all() and d[[1, 2]].isnan().all()
    empty = q[:0]
    y, k = B.qk_rope(empty, empty, pos[:0], table)
    assert y.shape == k.shape == (0, 2, 64)
    d, _, dg, _ = B.qk_rope_grad(empty, None, pos[:0], table, q=empty, q_gain=g)
    assert d.shape == (0, 2, 64) and torch.equal(dg, torch.zeros(64, device="cuda"))


@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", dict(factor=2.0)), ("llama3", dict(factor=8.0, low=1.0, high=4.0, original_max_pos=8192)),
                                        ("yarn", dict(factor=4.0, low=1.0, high=32.0, original_max_pos=4096))])
@pytest.mark.parametrize("rot,theta", [(64, 1e4), (128, 5e5), (32, 1e6)])
def test_rope_table(B, rot, theta, scaling, kw):
    """Far positions, against float64 frequencies written out here: an entry is
    one rounding of a cosine whose angle is within 2^-50 of itself."""
    n_pos = 200_000
    table = B.rope_table(n_pos, rot, theta, scaling, **kw).double().cpu()
    i = torch.arange(rot // 2, dtype=torch.float64)
    theta = float(np.float32(theta))
    w, m = theta ** (-2 * i / rot), 1.0
    if scaling == "linear":
        w = w / 2.0
    elif scaling == "llama3":
        wave = 2 * np.pi / w
        mid = (8192 / wave - 1.0) / 3.0
        w = torch.where(wave > 8192 / 1.0, w / 8, torch.where(wave < 8192 / 4.0, w, (1 - mid) * w / 8 + mid * w))
    elif scaling == "yarn":
        at = lambda t: rot * np.log(4096 / (t * 2 * np.pi)) / (2 * np.log(theta))  # noqa: E731
        lo, hi = max(np.floor(at(32.0)), 0), min(np.ceil(at(1.0)), rot - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        w, m = w / 4 * (1 - keep) + w * keep, 0.1 * np.log(4.0) + 1
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * w
    for j, f in ((0, torch.cos), (1, torch.sin)):
        want = f(a) * m
        T.assert_within(table[..., j], want, T.F * want.abs() + a * 2.0 ** -50 + 1e-12, "table")


# --------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------

def _attn_inputs(g, rows, hq, hk, hd, dt, std=1.0):
    qkv = _randn(g, rows, (hq + 2 * hk) * hd, dtype=dt, std=std)
    return (qkv[:, :hq * hd].unflatten(1, (hq, hd)), qkv[:, hq * hd:(hq + hk) * hd].unflatten(1, (hk, hd)),
            qkv[:, (hq + hk) * hd:].unflatten(1, (hk, hd)))


def _plan(B, section, column, offs, lens):
    return B.cod_plan(torch.from_numpy(section).cuda(), torch.from_numpy(column).cuda(), offs, torch.from_numpy(lens).cuda())


def _inside(offs, lens, rows):
    m = torch.zeros(rows, dtype=torch.bool)
    for o, n in zip(offs, lens):
        m[o:o + n] = True
    return m


def _check_attn(B, lengths, k_max, hq, hk, hd, dtype, r=0.7, r_min=0.2, std=1.0, scale=None, **pack):
    dt = T.DTYPES[dtype]
    section, column, offs, lens, rows = T.pack(lengths, k_max, r, r_min, **pack)
    say(f"[gpu] attention: columns {lengths[:8]} K={k_max} rows {rows} heads {hq}/{hk} x {hd} {dtype}")
    g = _gen(rows + hd + hq)
    q, k, v = _attn_inputs(g, rows, hq, hk, hd, dt, std)
    d_out = _randn(g, rows, hq, hd, dtype=dt)
    inside = _inside(offs, lens, rows)
    region = torch.zeros(rows, dtype=torch.bool)
    region[offs[0]:offs[-1]] = True
    # rows of no sample hold NaN, and must neither matter nor be written
    for t in (q, k, v, d_out):
        t[~inside.cuda()] = NAN
    plan = _plan(B, section, column, offs, lens)
    out = torch.full((rows, hq, hd), 7.0, device="cuda", dtype=dt)
    got = {"out": out}
    _, lse = B.cod_attn(q, k, v, plan, scale, out=out)
    got["lse"] = torch.full((hq, rows), -np.inf, device="cuda")
    got["lse"][:, :plan.rows] = lse
    outs = [torch.full(t.shape, 7.0, device="cuda", dtype=dt) for t in (q, k, v)]
    got["dq"], got["dk"], got["dv"] = B.cod_attn_grad(d_out, q, k, v, out, lse, plan, scale, dq=outs[0], dk=outs[1], dv=outs[2])
    ref = T.attn_ref(*(torch.where(inside[:, None, None].cuda(), t, 0) for t in (q, k, v)), section, column, offs, lens,
                     hd ** -0.5 if scale is None else scale, torch.where(inside[:, None, None].cuda(), d_out, 0))
    for name, (want, bound) in ref.items():
        x = got[name]
        if name == "lse":
            x = x[:, inside]
            want, bound = want[:, inside], bound[:, inside]
            assert torch.isneginf(lse.cpu()[:, (~inside & region)[:plan.rows]]).all()
        else:
            assert (x.cpu()[~region] == 7.0).all(), f"{name}: rows outside the regions were written"
            assert (x.cpu()[region & ~inside] == 0.0).all(), f"{name}: padding rows"
            x, want, bound = x[inside.cuda()], want[inside], bound[inside]
        T.assert_within(x, want, bound, name)
    return q, k, v, d_out, plan, got


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lengths,k_max,heads", [
    ([1], 1, (1, 1)), ([1, 1, 1], 8, (2, 1)), ([2], 3, (2, 2)), ([63], 1, (2, 1)), ([64, 65], 1, (2, 1)), ([127, 128, 129], 1, (1, 1)),
    ([40], 8, (4, 2)), ([17, 0, 33, 1, 0], 4, (2, 1)), ([100, 37], 8, (7, 1)), ([300], 8, (3, 3)), ([257, 90], 12, (4, 1)), ([70], 64, (2, 1))],
    ids=str)
def test_attention(B, lengths, k_max, heads, hd, dtype):
    _check_attn(B, lengths, k_max, *heads, hd, dtype, slack=3, lead=5, trail=2)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_many_query_heads_of_a_key_head(B, hd):
    """Groups that fill a wavefront's pairs, a workgroup's, and neither evenly."""
    for heads in ((33, 1), (64, 2), (130, 1)):
        _check_attn(B, [23, 6], 4, *heads, hd, "bf16", slack=1)


def test_strides_that_pass_32_bits(B):
    """Rows whose byte offsets pass 2^32: the results of the same rows close together."""
    g, hq, hk, hd = _gen(77), 4, 2, 64
    section, column, offs, lens, rows = T.pack([200, 400], 4)
    plan = _plan(B, section, column, offs, lens)
    wide = (1 << 32) // rows // 16 * 16 + 4096       # elements a row: the last half of the rows is past 2^32 bytes
    assert rows * wide * 2 > 1 << 33
    near = _attn_inputs(g, rows, hq, hk, hd, torch.bfloat16)
    d_out = _randn(g, rows, hq, hd, dtype=torch.bfloat16)
    big = torch.empty(rows, wide, device="cuda", dtype=torch.bfloat16)
    at = 0
    def place(t):
        nonlocal at
        n = t.shape[1] * hd
        view = big[:, at:at + n].unflatten(1, (t.shape[1], hd))
        at += n
        return view.copy_(t)
    far = [place(t) for t in near]
    out, lse = B.cod_attn(*near, plan)
    fout, flse = B.cod_attn(*far, plan, out=place(torch.zeros_like(near[0])))
    assert torch.equal(out, fout) and torch.equal(lse, flse)
    grads = B.cod_attn_grad(d_out, *near, out, lse, plan)
    fgrads = B.cod_attn_grad(place(d_out), *far, fout, flse, plan, dq=place(torch.zeros_like(near[0])),
                             dk=place(torch.zeros_like(near[1])), dv=place(torch.zeros_like(near[2])))
    assert all(torch.equal(a, b) for a, b in zip(grads, fgrads))
    table, gain = B.rope_table(512, hd, 1e4), 1 + _randn(g, hd, std=0.1)
    pos = torch.from_numpy(np.clip(column, 0, 511)).cuda()
    want = B.qk_rope(near[0], near[1], pos, table, "half", gain, gain)
    got = B.qk_rope(far[0], far[1], pos, table, "half", gain, gain, q_out=far[0], k_out=far[1])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    del big, far, fout, fgrads, got
    logits = torch.zeros(20_000, 128_256, device="cuda", dtype=torch.bfloat16)      # 5.1 GB
    logits[-3:] = _randn(g, 3, 128_256, dtype=torch.bfloat16)
    labels = torch.full((20_000,), -1, device="cuda", dtype=torch.int32)
    labels[-3:] = torch.tensor([5, 100_000, 128_255], device="cuda", dtype=torch.int32)
    want = B.cod_loss(logits[-3:].clone(), labels[-3:], None, 1)
    got = B.cod_loss(logits, labels, None, 1, d_logits=logits)
    assert torch.equal(want[0], got[0]) and torch.equal(want[2], got[2][-3:]) and torch.equal(want[3], logits[-3:])
    assert not logits[:-3].any()


def test_rope_gradient_of_no_key_heads(B):
    q, k = torch.ones(4, 2, 64, device="cuda"), torch.ones(4, 0, 64, device="cuda")
    pos, g = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    _, dk, dg, dgk = B.qk_rope_grad(q, k, pos, B.rope_table(8, 64, 1e4), q=q, k=k, q_gain=g, k_gain=g)
    assert dk.shape == (4, 0, 64) and dg.isfinite().all() and torch.equal(dgk, torch.zeros_like(g))


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_everything_kept(B, hd):
    """r = 1: every chain is K long (K = 64: chains longer than a wavefront's rows)."""
    _check_attn(B, [90], 64, 2, 1, hd, "f16", r=1.0)
    _check_attn(B, [150, 31], 5, 2, 1, hd, "bf16", r=1.0)


def test_attention_peaked_scores_and_scale(B):
    """Large scores (the softmax nearly picks one key), a negative and a zero scale."""
    _check_attn(B, [200], 8, 2, 1, 64, "f16", std=3.0)
    _check_attn(B, [100], 4, 2, 2, 128, "bf16", scale=-0.1)
    _check_attn(B, [100], 4, 2, 2, 64, "bf16", scale=0.0)


@pytest.mark.parametrize("hd", [64, 128])
def test_attention_many_short_samples(B, hd):
    rng = np.random.default_rng(4)
    _check_attn(B, [int(x) for x in rng.integers(0, 30, size=150)], 6, 2, 1, hd, "bf16", slack=1)


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "f16")])
def test_attention_long_sample(B, hd, dtype):
    _check_attn(B, [1300, 5], 8, 2, 1, hd, dtype)


def test_attention_layouts_and_runs_agree(B):
    """Head-major tensors, padded rows and a second run give the same bits."""
    q, k, v, d_out, plan, got = _check_attn(B, [130, 60], 8, 4, 2, 64, "bf16")
    section = None
    again, lse = B.cod_attn(q, k, v, plan)
    assert torch.equal(again, got["out"])
    hm = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    wide = lambda t: torch.full((t.shape[0], t.shape[1] + 1, t.shape[2] + 8), NAN, device="cuda", dtype=t.dtype)[:, 1:, :t.shape[2]].copy_(t)  # noqa: E731
    for how in (hm, wide):
        o, l2 = B.cod_attn(how(q), how(k), how(v), plan, out=how(torch.zeros_like(q)))
        assert torch.equal(o, got["out"]) and torch.equal(l2, lse)
        grads = B.cod_attn_grad(how(d_out), how(q), how(k), how(v), how(o), l2, plan, dq=how(q * 0), dk=how(k * 0), dv=how(v * 0))
        for name, t in zip(("dq", "dk", "dv"), grads):
            assert torch.equal(t, got[name]), name
    del section


def test_plan_turns_away_rows_in_another_form(B):
    """Checked on the device and reported by the call: the plan is not set."""
    section, column, offs, lens, rows = T.pack([20, 30], 4)
    _plan(B, section, column, offs, lens)

    def refused(sec=section, col=column, n=lens):
        with pytest.raises(B.PardError) as e:
            _plan(B, sec, col, offs, n)
        assert e.value.status == B.PARD_ERR_ARG
    at = int(offs[1])
    for i, k, j in ((0, 0, 0), (3, 65, 5), (at + 2, 1, 9), (at + len(section) // 3, 2, 8191), (at - 1, 4, 1), (5, 1, -3),
                    (at - 1, 2, 2 ** 31 - 1), (at - 1, 2 ** 31 - 1, 4), (at - 1, -2 ** 31, 4)):
        s, c = section.copy(), column.copy()
        s[i], c[i] = k, j
        refused(s, c)
    s, c = section.copy(), column.copy()
    s[at - 1], c[at - 1] = s[at - 2], c[at - 2]      # a row twice
    refused(s, c)
    refused(n=np.array([lens[0] + 1, lens[1]], np.int32))
    refused(n=np.array([-1, lens[1]], np.int32))


def test_attention_of_no_rows(B):
    plan = B.cod_plan(torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), [0, 0, 0],
                      torch.zeros(2, dtype=torch.int32, device="cuda"))
    q = torch.zeros(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    out, lse = B.cod_attn(q, q, q, plan)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    assert all(t.shape == (0, 2, 64) for t in B.cod_attn_grad(q, q, q, q, out, lse, plan))


# --------------------------------------------------------------------------
# the loss
# --------------------------------------------------------------------------

def _loss_inputs(g, rows, vocab, k_max, dt, std=2.0):
    logits = _randn(g, rows, vocab, dtype=dt, std=std)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    section = torch.randint(1, k_max + 1, (rows,), generator=g, device="cuda").to(torch.int32)
    return logits, labels, section


def _check_loss(logits, labels, section, k_max, weights, scale, got):
    loss, parts, rows, d, e_row, e_d = T.loss_ref(logits, labels, section, k_max, weights, scale)
    T.assert_within(got[2], rows, e_row, "row losses")
    # means: of float32 row losses in float64, rounded once
    mean_bound = float(e_row.max()) if len(e_row) else 0.0
    T.assert_within(got[1], parts, mean_bound + T.F * parts.abs(), "subtask means")
    wsum = 1.0 if weights is None else sum(abs(w) for w in weights)
    T.assert_within(got[0], loss, torch.as_tensor(wsum * mean_bound + 2 * T.F * wsum * float(parts.abs().max() if len(parts) else 0)), "loss")
    if got[3] is not None:
        T.assert_within(got[3], d, e_d, "gradient")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,k_max", [(1, 1, 1), (3, 2, 2), (7, 63, 3), (50, 1024, 4), (5, 50257, 8), (3, 128256, 8), (2, 152064, 2),
                                              (130, 999, 64), (4, 300001, 2), (1, 8193, 1), (300, 17, 1)])
def test_loss(B, rows, vocab, k_max, dtype):
    g, dt = _gen(rows + vocab), T.DTYPES[dtype]
    say(f"[gpu] loss {rows} x {vocab} K={k_max} {dtype}")
    logits, labels, section = _loss_inputs(g, rows, vocab, k_max, dt)
    scale = 512.0 if dtype == "f16" else 1.5
    for weights in (None, [0.5 + 0.25 * k for k in range(k_max)]):
        got = B.cod_loss(logits, labels, section, k_max, weights, grad_scale=scale)
        _check_loss(logits, labels, section, k_max, weights, scale, got)
        plain = B.cod_loss(logits, labels, section, k_max, weights, grad=False)
        # (not bit for bit the same: without a gradient a row's terms are added in
        # another order, and each order's roundings, which the row's bound counts,
        # are others)
        assert plain[3] is None
        _check_loss(logits, labels, section, k_max, weights, scale, plain)


def test_loss_rows_that_do_not_count(B):
    """Labels below 0, subtasks outside 1..K, a subtask without rows; no counted row."""
    g = _gen(8)
    logits, labels, section = _loss_inputs(g, 40, 333, 3, torch.float32)
    section[section == 2] = 1
    labels[::3] = -100
    section[1::7], section[2::7] = 0, 4
    logits[0] = NAN                                  # (does not count)
    ref = logits.clone()
    ref[0] = 0
    for weights in (None, [1.0, 5.0, 0.5]):
        got = B.cod_loss(logits, labels, section, 3, weights)
        _check_loss(ref, labels, section, 3, weights, 1.0, got)
        assert got[1][1] == 0.0 and (got[3][0] == 0).all()
    got = B.cod_loss(logits, torch.full_like(labels, -1), section, 3)
    assert float(got[0]) == 0.0 and (got[1] == 0).all() and (got[2] == 0).all() and (got[3] == 0).all()
    got = B.cod_loss(logits[:0], labels[:0], section[:0], 3)
    assert float(got[0]) == 0.0 and (got[1] == 0).all() and got[3].shape == (0, 333)


def test_loss_extremes(B):
    """Masked logits (-inf and the type's lowest), large ones, a +inf or NaN row, a label past the vocabulary."""
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        g = _gen(9)
        logits, labels, _ = _loss_inputs(g, 6, 5000, 1, dt)
        labels.clamp_(min=2000)
        logits[0, :1999] = -float("inf")
        logits[1, :1999] = torch.finfo(dt).min
        logits[2] += 50.0 if dt != torch.float16 else 20.0
        ref = logits.clone()
        got = B.cod_loss(logits, labels, None, 1)
        loss, _, rows, d, e_row, e_d = T.loss_ref(ref.float().double(), labels, torch.ones_like(labels), 1, None, 1.0)
        top = ref.float().clamp(min=-100).abs().amax(-1).double().cpu()      # (terms at -100 and below are 0)
        _, _, _, _, e_row, e_d = T.loss_ref(ref.float().clamp(min=-100).to(dt), labels, torch.ones_like(labels), 1, None, 1.0)
        T.assert_within(got[2], rows, e_row + 0 * top, "row losses")
        T.assert_within(got[3], d, e_d, "gradient")
        logits[3, 7], logits[4, 8] = float("inf"), NAN
        labels[5] = 5000
        got = B.cod_loss(logits, labels, None, 1)
        assert got[2][:3].isfinite().all() and not got[2][3:].isfinite().any() and not got[0].isfinite()
        assert got[3][:3].isfinite().all() and got[3][3, 7].isnan() and got[3][4].isnan().all() and got[3][5].isnan().all()


def test_loss_of_rows_at_the_ends_of_the_type(B):
    """Rows masked everywhere with the type's lowest value, or everywhere but at
    one logit; the largest value; -inf next to NaN, which no row loses."""
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        for vocab in (5, 1000, 9001, 200_000):       # (with and without rows in registers)
            low, top = torch.finfo(dt).min, torch.finfo(dt).max
            logits = torch.full((5, vocab), low, device="cuda", dtype=dt)
            logits[1, vocab // 2] = 0.5
            logits[2] = top
            logits[3] = -float("inf")
            logits[3, 1:3] = top
            logits[4] = -float("inf")
            logits[4, vocab - 2] = NAN
            labels = torch.tensor([vocab - 1, vocab // 2, 0, 2, 1], dtype=torch.int32, device="cuda")
            got = B.cod_loss(logits, labels, None, 1)
            # ce: m - x is 0 in every row; the logarithm of the sum, its sum and
            # product: (vocab + 8) roundings of float32
            n = torch.tensor([vocab, 1, vocab, 2], dtype=torch.float64)
            T.assert_within(got[2][:4], n.log(), (vocab + 8) * T.F * (1 + n.log()), "row losses")
            p = torch.zeros(4, vocab, dtype=torch.float64)
            p[0], p[1, vocab // 2], p[2], p[3, 1:3] = 1 / vocab, 1.0, 1 / vocab, 0.5
            d = p.clone()
            d[torch.arange(4), labels[:4].long().cpu()] -= 1
            d /= 5
            T.assert_within(got[3][:4], d, T.unit(dt) * d.abs() + (vocab + 16) * T.F * (p + d.abs()) + T.floor_of(dt), "gradient")
            assert got[2][4].isnan() and got[3][4].isnan().all()
            plain = B.cod_loss(logits, labels, None, 1, grad=False)
            T.assert_within(plain[2][:4], n.log(), (vocab + 8) * T.F * (1 + n.log()), "row losses alone")
            assert plain[2][4].isnan()


def test_loss_in_place_and_strided(B):
    g = _gen(10)
    for dt, vocab in ((torch.bfloat16, 4099), (torch.float32, 1024), (torch.float16, 152064)):
        logits, labels, section = _loss_inputs(g, 9, vocab, 2, dt)
        want = B.cod_loss(logits, labels, section, 2)
        wide = torch.full((9, vocab + 5), NAN, device="cuda", dtype=dt)
        wide[:, 2:2 + vocab] = logits
        part = wide[:, 2:2 + vocab]
        say(f"[gpu] loss in place, {vocab} {dt}")
        got = B.cod_loss(part, labels, section, 2, d_logits=part)
        T.assert_within(got[2], want[2].double().cpu(), 1e-5 * want[2].abs().double().cpu(), "row losses")
        _check_loss(logits, labels, section, 2, None, 1.0, (got[0], got[1], got[2], part))
        assert wide[:, :2].isnan().all() and wide[:, 2 + vocab:].isnan().all()


@pytest.mark.parametrize("dtype,rows,vocab", [("bf16", 2500, 40), ("f16", 2049, 2000), ("f32", 300, 4100), ("bf16", 270, 40_001),
                                              ("f32", 4500, 33), ("bf16", 9000, 40), ("f32", 8300, 700), ("f32", 4200, 3001),
                                              ("f32", 2100, 5002), ("f32", 1100, 9003), ("f32", 530, 20_001), ("f32", 260, 40_003),
                                              ("f16", 258, 150_001)])
def test_loss_more_rows_than_workgroups(B, dtype, rows, vocab):
    """Rows that a workgroup takes after its first, with gradients in tensors at
    another place in 16 bytes, and without."""
    dt = T.DTYPES[dtype]
    g = _gen(rows)
    logits, labels, section = _loss_inputs(g, rows, vocab, 5, dt)
    got = B.cod_loss(logits, labels, section, 5)
    _check_loss(logits, labels, section, 5, None, 1.0, got)
    off = torch.full((rows * (vocab + 3) + 1,), NAN, device="cuda", dtype=dt)[1:].view(rows, vocab + 3)
    other = B.cod_loss(logits, labels, section, 5, d_logits=off[:, :vocab])
    _check_loss(logits, labels, section, 5, None, 1.0, other)
    assert off[:, vocab:].isnan().all()
    plain = B.cod_loss(logits, labels, section, 5, grad=False)
    _check_loss(logits, labels, section, 5, None, 1.0, (*plain[:3], got[3]))


# --------------------------------------------------------------------------
# together
# --------------------------------------------------------------------------

def _step_inputs(B, hd=64, dt=torch.bfloat16, k_max=4, vocab=515, seed=21):
    """Real COD data of the library, and one layer's tensors."""
    rng = np.random.default_rng(seed)
    lengths = [2, 40, 131, 9]
    offs = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    tokens = torch.from_numpy(rng.integers(0, vocab - 1, size=int(offs[-1])).astype(np.int32)).cuda()
    out_offs, out, lens = B.cod_build(tokens, offs, k_max, 0.7, 0.2, vocab - 1, seed)
    g = _gen(seed)
    rows = int(out_offs[-1])
    valid = _inside(out_offs, lens.cpu().numpy(), rows).cuda()
    pos, labels = torch.where(valid, out["pos"], 0).to(torch.int32), torch.where(valid, out["labels"], -1).to(torch.int32)
    section, column = out["section"], out["column"]
    x = dict(qkv=_randn(g, rows, 8 * hd, dtype=dt), w=_randn(g, 4 * hd, vocab, dtype=dt, std=0.05), gq=1 + _randn(g, hd, std=0.1),
             gk=1 + _randn(g, hd, std=0.1))
    return x, pos, labels, section, column, out_offs, lens, valid


def _step(B, x, pos, table, labels, section, plan, k_max, hd=64):
    """Rotation, attention, output product, loss, and back to the projections."""
    q, k, v = (t.unflatten(1, (-1, hd)) for t in (x["qkv"][:, :4 * hd], x["qkv"][:, 4 * hd:6 * hd], x["qkv"][:, 6 * hd:]))
    rq, rk = B.qk_rope(q, k, pos, table, "half", x["gq"], x["gk"])
    out, lse = B.cod_attn(rq, rk, v, plan)
    logits = out.flatten(1) @ x["w"]
    loss, parts, rows, d_logits = B.cod_loss(logits, labels, section, k_max, [1.0] * k_max, grad_scale=64.0)
    d_out = (d_logits @ x["w"].T.contiguous()).unflatten(1, (4, hd))
    dq, dk, dv = B.cod_attn_grad(d_out, rq, rk, v, out, lse, plan)
    dxq, dxk, dgq, dgk = B.qk_rope_grad(dq, dk, pos, table, "half", q, k, x["gq"], x["gk"])
    return dict(loss=loss, parts=parts, rows=rows, dq=dxq, dk=dxk, dv=dv, dgq=dgq, dgk=dgk)


def test_a_training_step_against_autograd(B):
    """cod_build's rows through all operators, against float64 autograd.  Seven
    roundings to the stored type lie between an input and its gradient (rotated
    heads, probabilities, output, logits, their gradient, the output's, the score
    gradients', and the result): in the 2-norm each adds at most u of the terms it
    sums, whose norm cancellation makes up to a few times the result's: 16 u."""
    k_max, hd = 4, 64
    for dt in (torch.bfloat16, torch.float16):
        x, pos, labels, section, column, offs, lens, valid = _step_inputs(B, hd, dt, k_max)
        table = B.rope_table(256, hd, 1e4)
        plan = B.cod_plan(section, column, offs, lens)
        got = _step(B, x, pos, table, labels, section, plan, k_max)
        y = {n: t.double().cpu().requires_grad_(n != "w") for n, t in x.items()}
        q, k, v = (t.unflatten(1, (-1, hd)) for t in (y["qkv"][:, :4 * hd], y["qkv"][:, 4 * hd:6 * hd], y["qkv"][:, 6 * hd:]))
        cs = table.double().cpu()[pos.long().cpu()][:, None]
        norm = lambda t, g: T.turn(t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * g, cs[..., 0], cs[..., 1], "half")  # noqa: E731
        rq, rk = norm(q, y["gq"]), norm(k, y["gk"])
        total, sec, col = 0.0, section.cpu().numpy(), column.cpu().numpy()
        ces, secs = [], []
        for o, n in zip(offs, lens.cpu().numpy()):
            sl = slice(int(o), int(o) + int(n))
            seen = T.seen_mask(sec[sl], col[sl])
            heads = [torch.softmax((rq[sl, h] @ rk[sl, h // 2].T * hd ** -0.5).masked_fill(~seen, -np.inf), -1) @ v[sl, h // 2] for h in range(4)]
            logits = torch.cat(heads, -1) @ y["w"]
            ces.append(torch.nn.functional.cross_entropy(logits, labels.long().cpu()[sl], reduction="none"))
            secs.append(torch.from_numpy(sec[sl]).long())
        ce, secs = torch.cat(ces), torch.cat(secs)
        total = sum(ce[secs == s].mean() for s in range(1, k_max + 1))
        d = dict(zip(("qkv", "gq", "gk"), torch.autograd.grad(64.0 * total, (y["qkv"], y["gq"], y["gk"]))))
        u = T.unit(dt)
        far = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())  # noqa: E731
        assert abs(float(got["loss"]) - float(total.detach())) < 16 * u * float(total.detach())
        keep = valid.cpu()
        for name, a, b in (("dq", got["dq"], d["qkv"][:, :4 * hd]), ("dk", got["dk"], d["qkv"][:, 4 * hd:6 * hd]), ("dv", got["dv"], d["qkv"][:, 6 * hd:])):
            e = far(a.flatten(1)[valid], b[keep])
            say(f"[gpu] step {dt} {name}: {e:.2e} ({e / u:.1f} u)")
            assert e < 16 * u, name
        assert far(got["dgq"], d["gq"]) < 16 * u and far(got["dgk"], d["gk"]) < 16 * u


def test_a_captured_step_on_another_stream(B):
    """The whole step captured into a graph on a stream of its own, replayed with
    other inputs between eager steps: every replay equals the eager step's bits."""
    k_max, hd = 4, 64
    x, pos, labels, section, column, offs, lens, valid = _step_inputs(B)
    x = {n: t.clone() for n, t in x.items()}
    table = B.rope_table(256, hd, 1e4)
    plan = B.cod_plan(section, column, offs, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(B, x, pos, table, labels, section, plan, k_max)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = _step(B, x, pos, table, labels, section, plan, k_max)
    for turn in range(4):
        say(f"[gpu] replay {turn}")
        x["qkv"].copy_(_randn(_gen(100 + turn), *x["qkv"].shape, dtype=torch.bfloat16))
        want = {n: t.clone() for n, t in _step(B, x, pos, table, labels, section, plan, k_max).items()}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in want.items():
            assert torch.equal(got[n][valid] if n in ("dq", "dk", "dv", "rows") else got[n], t[valid] if n in ("dq", "dk", "dv", "rows") else t), (turn, n)


def test_two_streams_at_once(B):
    """Steps enqueued on two streams without waiting between them."""
    k_max, hd = 4, 64
    table = B.rope_table(256, hd, 1e4)
    sets = [_step_inputs(B, seed=s) for s in (31, 32)]
    plans = [B.cod_plan(s[3], s[4], s[5], s[6]) for s in sets]
    want = [_step(B, s[0], s[1], table, s[2], s[3], p, k_max) for s, p in zip(sets, plans)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = _step(B, sets[i][0], sets[i][1], table, sets[i][2], sets[i][3], plans[i], k_max)
    torch.cuda.synchronize()
    for i in (0, 1):
        v = sets[i][7]
        for n, t in want[i].items():
            assert torch.equal(got[i][n][v] if n in ("dq", "dk", "dv", "rows") else got[i][n], t[v] if n in ("dq", "dk", "dv", "rows") else t), (i, n)


def test_the_stream_argument(B):
    g = _gen(1)
    table = B.rope_table(64, 64, 1e4)
    q, pos = _randn(g, 50, 2, 64), torch.arange(50, device="cuda", dtype=torch.int32)
    want, _ = B.qk_rope(q, None, pos, table)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, _ = B.qk_rope(q, None, pos, table, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
