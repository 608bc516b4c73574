"""GPU checks of the serving operators (a paged cache, attention over it, logits
before tokens are picked) against plain float64 forms, element by element within
derived bounds (serve_common); what is stored is compared exactly."""
import numpy as np
import pytest
import torch

import serve_common as S
import train_common as T
from gpu_common import require_gpu, say

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    require_gpu()
    from paper_2504_18583_amd import binding
    return binding


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _cache(B, n_pages, page, hk, hd, kind):
    """A cache whose every byte is set, to NaN where it can be."""
    c = B.kv_cache(n_pages, page, hk, hd, T.DTYPES.get(kind, kind))
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            t.fill_(255 if t.dtype == torch.uint8 else NAN)
    return c


def _values(c, kind, name, pages, places):
    x = getattr(c, name)[pages.cuda(), :, places.cuda()]
    if kind in S.BITS:
        return S.decoded(x, getattr(c, name + "_scale")[pages.cuda(), :, places.cuda()], kind)
    return x.double().cpu()


# --------------------------------------------------------------------------
# the cache
# --------------------------------------------------------------------------

CACHE_SHAPES = [([1], [0], 16, 1, 64), ([3, 0, 17], [15, 9, 30], 16, 2, 64), ([40, 1, 7, 0], [0, 63, 64, 2], 64, 8, 128),
                ([5] * 9, list(range(9)), 32, 3, 64), ([300, 2], [1, 255], 256, 5, 128), ([2], [4095], 4096, 1, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("shape", CACHE_SHAPES, ids=str)
def test_write_and_read(B, shape, kind, dtype):
    rows, past, page, hk, hd = shape
    say(f"[gpu] cache {shape} {kind} of {dtype}")
    dt, g = T.DTYPES[dtype], _gen(sum(rows) + hd)
    batch = S.Batch(rows, past, page, lead=2, trail=3)
    c, on = _cache(B, batch.n_pages, page, hk, hd, kind), batch.device(B)
    kv = _randn(g, batch.n, 2 * hk * hd, dtype=dt) * torch.exp2(torch.randint(-12, 6, (batch.n, 1), generator=g, device="cuda")).to(dt)
    k, v = kv[:, :hk * hd].unflatten(1, (hk, hd)), kv[:, hk * hd:].unflatten(1, (hk, hd))
    before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]
    B.kv_write(k, v, c, on)
    touched = torch.zeros(batch.n_pages, page, dtype=torch.bool)
    for s in range(len(rows)):
        if not rows[s]:
            continue
        pages, places = batch.places(s, past[s] + np.arange(rows[s]))
        touched[pages, places] = True
        for name, x in (("k", k), ("v", v)):
            x = x[list(batch.seq_rows(s))]
            want = S.stored(x, kind) if kind in S.BITS else x.to(T.DTYPES[kind]).double().cpu()
            assert torch.equal(_values(c, kind, name, pages, places), want), (s, name)
    for t, old in zip([t for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None], before):
        m = ~touched.cuda()[:, None].expand(t.shape[:3])
        assert torch.equal(t[m].view(torch.uint8), old[m].view(torch.uint8)), "a place that is no row's was written"
    # back, into given tensors of each type: rows of no sequence stay
    inside = batch.owned().cuda()
    for out in ("bf16", "f16", "f32"):
        ko, vo = (torch.full((batch.n, hk, hd), 7.0, device="cuda", dtype=T.DTYPES[out]) for _ in "kv")
        got = B.kv_read(c, on, batch.n, k_out=ko, v_out=vo)
        assert got[0] is ko and got[1] is vo
        for o, x in ((ko, k), (vo, v)):
            want = S.stored(x, kind) if kind in S.BITS else x.to(T.DTYPES[kind]).double().cpu()
            assert torch.equal(o[inside].cpu(), want.to(T.DTYPES[out])[inside.cpu()]) and bool((o[~inside] == 7).all())
    new = B.kv_read(c, on, batch.n)
    assert new[0].dtype == torch.bfloat16 and torch.equal(new[1][inside].float(), vo[inside].to(torch.bfloat16).float())


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_blocks_at_their_borders(B, kind):
    """Ties, the largest value of each scale and what is next to it, tiny and huge
    blocks, zeros of both signs, NaN and infinities in one block of a head."""
    hd, top = 64, S.BITS[kind][2]
    g = S.grid(kind)
    mid = (g[1:] + g[:-1]) / 2
    rows = []
    for e in (-140, -127, -126, -120, -20, 0, 3, 100, 118):
        for lead in (top, top * (1 + 2.0 ** -20), top * (1 - 2.0 ** -20), top / 2, 2.0 ** -10):
            for part in range(0, len(mid), 31):
                m = mid[part:part + 31]
                block = torch.zeros(32, dtype=torch.float64)
                block[:len(m)] = m * (-1.0) ** torch.arange(len(m))
                block[31] = lead
                rows.append(torch.cat([block, block.flip(0)]) * 2.0 ** e)
    x = torch.stack(rows).float()
    extra = torch.zeros(5, 64)
    extra[1] = -0.0
    extra[2, 3], extra[3, 40], extra[4, 31] = NAN, INF, -INF
    x = torch.cat([x, extra]).cuda()[:, None]
    batch = S.Batch([len(x)], [0], 16)
    c = _cache(B, batch.n_pages, 16, 1, hd, kind)
    B.kv_write(x, -x, c, batch.device(B))
    k, v = B.kv_read(c, batch.device(B), len(x), torch.float32)
    for got, src in ((k, x), (v, -x)):
        want = S.stored(src, kind)
        assert torch.equal(got.cpu().double().nan_to_num(123.0), want.nan_to_num(123.0))
    # the other block of a head with a NaN keeps its values
    assert k[-3, 0, 32:].isfinite().all() and k[-3, 0, :32].isnan().all() and k[-2, 0, :32].isfinite().all() and k[-2, 0, 32:].isnan().all()


def test_rows_without_a_place_and_odd_strides(B):
    """Positions below 0, past the table, pages outside the cache; rows at odd
    element offsets, which no 16-byte access fits; a row or head for all."""
    g = _gen(4)
    table = torch.tensor([[1, 9, -1], [2, 0, 3]], dtype=torch.int32, device="cuda")
    start, kv_len = torch.tensor([0, 6, 10], dtype=torch.int32, device="cuda"), torch.tensor([4, 50], dtype=torch.int32, device="cuda")
    on = B.KVBatch(table, start, kv_len)            # rows at positions -2 .. 3 and 46 .. 49 (the table ends at 48)
    for kind in ("bf16", "e4m3", "e2m1"):
        say(f"[gpu] odd rows {kind}")
        c = _cache(B, 4, 16, 2, 64, kind)
        raw = _randn(g, 10 * 259 + 1, dtype=torch.bfloat16)
        k = raw[1:].view(10, 259)[:, :128].unflatten(1, (2, 64))
        v = _randn(g, 10, 1, 64, dtype=torch.bfloat16).expand(10, 2, 64)
        B.kv_write(k, v, c, on)
        out = torch.full((10 * 259 + 1,), 7.0, device="cuda")[1:].view(10, 259)[:, :128].unflatten(1, (2, 64))
        got = B.kv_read(c, on, 10, k_out=out, v_out=torch.empty(2, 10, 64, device="cuda").transpose(0, 1))
        there = torch.tensor([0, 0, 1, 1, 1, 1, 1, 1, 0, 0], dtype=torch.bool)
        for o, x in zip(got, (k, v)):
            want = S.stored(x, kind) if kind in S.BITS else x.double().cpu()
            assert torch.equal(o.cpu().double()[there], want[there]) and o.cpu()[~there].isnan().all()
        # pages that the table does not reach through a valid entry are as they were
        held = c.k.view(torch.uint8)[0]
        assert bool((held == held[0, 0]).all()) if kind != "bf16" else bool(c.k[0].isnan().all())
    # row 3 of sequence 0's second page: an entry outside the cache
    kv_len[0] = 20
    k, v = B.kv_read(c, on, 10, torch.float32)
    assert k[2:6].isnan().all() and v[2:6].isnan().all()
    none = B.kv_read(c, on, 0)
    assert none[0].shape == (0, 2, 64)


# --------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------

def _check_attn(B, rows, past, page, hq, hk, hd, dtype, kind, window=0, sinks=0, std=1.0, scale=None, known=False, lead=0, trail=0, seed=0):
    dt = T.DTYPES[dtype]
    say(f"[gpu] attention: rows {rows[:6]} past {past[:6]} page {page} heads {hq}/{hk} x {hd} {dtype} cache {kind} window {window}+{sinks}")
    g = _gen(sum(rows) + hd + hq + seed)
    batch = S.Batch(rows, past, page, window, sinks, lead=lead, trail=trail, seed=seed)
    c = _cache(B, batch.n_pages, page, hk, hd, kind)
    # what the rows see, and nothing else
    held = {}
    for s in range(len(rows)):
        if not rows[s]:
            continue
        j, _ = batch.seen(s)
        pages, places = batch.places(s, j)
        k, v = _randn(g, len(j), hk, hd, dtype=dt, std=std), _randn(g, len(j), hk, hd, dtype=dt)
        if kind in S.BITS:
            # every position as the one row of a sequence of its own, a page long
            B.kv_write(k, v, c, B.KVBatch(pages[:, None].to(torch.int32).cuda(), torch.arange(len(j) + 1, dtype=torch.int32, device="cuda"),
                                          (places + 1).to(torch.int32).cuda()))
            held[s] = [S.stored(x, kind).to(dt).double() for x in (k, v)]
        else:
            c.k[pages.cuda(), :, places.cuda()], c.v[pages.cuda(), :, places.cuda()] = k, v
            held[s] = [k.double().cpu(), v.double().cpu()]
    q = _randn(g, batch.n, hq, hd, dtype=dt, std=std)
    q[~batch.owned().cuda()] = NAN
    out = torch.full((batch.n, hq, hd), 7.0, device="cuda", dtype=dt)
    got, lse = B.kv_attn(q, c, batch.device(B, max(rows) if known else 0), scale, window, sinks, out=out)
    again = B.kv_attn(q, c, batch.device(B, max(rows) if known else 0), scale, window, sinks)
    ref = S.attn_ref(q.nan_to_num(0.0), lambda s, j: held[s][0], lambda s, j: held[s][1], batch, hd ** -0.5 if scale is None else scale)
    inside = batch.owned()
    T.assert_within(got[inside.cuda()], ref["out"][0][inside], ref["out"][1][inside], "out")
    T.assert_within(lse[:, inside.cuda()], ref["lse"][0][:, inside], ref["lse"][1][:, inside], "lse")
    assert bool((got[~inside.cuda()] == 7).all()), "a row of no sequence was written"
    assert torch.equal(again[0][inside.cuda()], got[inside.cuda()]) and torch.equal(again[1][:, inside.cuda()], lse[:, inside.cuda()])


ATTN = [  # rows, past, page, heads, key heads, head_dim
    ([1], [0], 16, 1, 1, 64), ([1], [63], 16, 4, 2, 64), ([1], [64], 16, 8, 1, 128), ([1, 1, 1], [14, 15, 16], 16, 2, 1, 64),
    ([9, 9], [100, 31], 32, 8, 2, 128), ([9, 0, 4, 1], [7, 50, 0, 129], 16, 14, 2, 64), ([5], [511], 64, 5, 5, 128), ([13, 2], [900, 1500], 128, 28, 4, 128),
    ([33], [0], 16, 3, 1, 64), ([64, 65, 63], [1, 0, 200], 256, 4, 4, 64), ([130], [70], 16, 8, 8, 128), ([200, 1], [300, 1023], 32, 32, 8, 64),
    ([1], [2], 16, 40, 1, 64), ([3], [5], 16, 100, 1, 128), ([1] * 70, [(7 * i) % 90 for i in range(70)], 16, 2, 2, 64), ([1], [4000], 4096, 4, 1, 128)]


@pytest.mark.parametrize("dtype,kind", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "e2m1"), ("f16", "e2m1")])
@pytest.mark.parametrize("shape", ATTN, ids=lambda s: f"{s[0][:3]}-{s[1][:3]}-{s[2:]}")
def test_attention(B, shape, dtype, kind):
    rows, past, page, hq, hk, hd = shape
    _check_attn(B, rows, past, page, hq, hk, hd, dtype, kind, lead=1, trail=2)


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (17, 4), (64, 4), (100, 16), (100, 17), (33, 300), (1000, 4), (5, 100000)])
def test_attention_within_a_window(B, window, sinks, kind):
    for hd, hq, hk, page in ((64, 4, 2, 16), (128, 8, 2, 32)):
        _check_attn(B, [1, 9, 40, 0, 150], [0, 257, 500, 9, 333], page, hq, hk, hd, "bf16", kind, window, sinks, known=hd == 64)


@pytest.mark.parametrize("scale,std", [(None, 8.0), (0.0, 1.0), (-0.2, 1.0), (4.0, 1.0)])
def test_attention_scales(B, scale, std):
    """Peaked softmaxes, no scale, a negative one."""
    for rows, past in (([1, 9], [300, 40]), ([150], [77])):
        _check_attn(B, rows, past, 16, 8, 2, 64, "bf16", "bf16", std=std, scale=scale)
        _check_attn(B, rows, past, 16, 8, 2, 128, "f16", "e4m3", std=std, scale=scale)


@pytest.mark.parametrize("known", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_attention_of_ragged_batches(B, kind, known):
    """Single tokens beside chunks, long contexts beside short ones (split over
    workgroups and joined), and many sequences."""
    _check_attn(B, [1, 70, 1, 1, 9], [5000, 1000, 30, 0, 2600], 16, 8, 2, 64, "bf16", kind, known=known)
    _check_attn(B, [1] * 30 + [300], [17 * i for i in range(30)] + [900], 64, 8, 2, 128, "bf16", kind, known=known)
    _check_attn(B, [1 + i % 3 for i in range(300)], [i % 40 for i in range(300)], 16, 4, 2, 64, "bf16", kind, known=known)
    _check_attn(B, [2] * 1100, [i % 23 for i in range(1100)], 16, 2, 1, 64, "bf16", kind, known=known)
    _check_attn(B, [1], [20000], 64, 8, 1, 128, "bf16", kind, known=known)
    _check_attn(B, [9], [9000], 16, 16, 4, 64, "bf16", kind, known=known)
    _check_attn(B, [70], [8000], 16, 4, 2, 64, "bf16", kind, known=known)


@pytest.mark.parametrize("rows", [1, 7, 12, 40])
def test_attention_of_many_sequences_with_long_ones_among_them(B, rows):
    """More sequences than a wavefront has lanes (their running numbers come from a
    launch ahead), some of them split: every size of tile."""
    n = 200
    long = {3: 9000, 64: 4000, 150: 2500, 199: 7000}
    for kind in ("bf16", "e4m3"):
        _check_attn(B, [rows if i % 5 else 0 for i in range(n - 1)] + [rows], [long.get(i, i % 29) for i in range(n)], 16, 8, 2, 64, "bf16", kind,
                    known=kind == "bf16", lead=3, trail=2)
    _check_attn(B, [1] * 90 + [rows * 9], [i % 50 for i in range(90)] + [5000], 32, 8, 2, 128, "bf16", "bf16", known=True)
    _check_attn(B, [rows] * 70, [i % 90 + 3 * 600 * (i == 66) for i in range(70)], 16, 4, 1, 64, "f16", "e2m1", 300, 20)


def test_a_wrong_hint_changes_no_result(B):
    """max_seq_rows below and above the truth."""
    g = _gen(1)
    batch = S.Batch([40, 1, 7], [20, 300, 90], 16)
    c = B.KVCache(*(_randn(g, batch.n_pages, 2, 16, 64, dtype=torch.bfloat16) for _ in "kv"))
    q = _randn(g, batch.n, 8, 64, dtype=torch.bfloat16)
    K = lambda x: lambda s, j: x.double().cpu()[batch.places(s, j)[0], :, batch.places(s, j)[1]]  # noqa: E731
    ref = S.attn_ref(q, K(c.k), K(c.v), batch, 0.125)
    for hint in (0, 1, 3, 40, 1000, 2 ** 31 - 1):
        say(f"[gpu] hint {hint}")
        out, lse = B.kv_attn(q, c, batch.device(B, hint))
        T.assert_within(out, *ref["out"], f"out {hint}")
        T.assert_within(lse, *ref["lse"], f"lse {hint}")


@pytest.mark.parametrize("rows", [1, 5, 150])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_rows_that_see_nothing_and_positions_without_a_page(B, kind, rows):
    """A negative position: 0 and -inf.  A page outside the cache, or past the
    table: NaN in the rows that see it, and in no other."""
    g = _gen(rows)
    hq, hk, hd, page = 4, 2, 64, 16
    table = torch.arange(40, dtype=torch.int32).repeat(3, 1)
    table[1, 2] = 40                                 # positions 32 .. 47 of sequence 1
    start = torch.tensor([0, rows, 2 * rows, 3 * rows], dtype=torch.int32)
    kv_len = torch.tensor([rows - 3 if rows > 3 else 0, 30 + rows, 40 * 16 + rows // 2], dtype=torch.int32)
    c = _cache(B, 40, page, hk, hd, kind)
    x = _randn(g, 640, hk, hd, dtype=torch.bfloat16)
    whole = B.KVBatch(table[:1].contiguous().cuda(), torch.tensor([0, 640], dtype=torch.int32, device="cuda"), torch.tensor([640], dtype=torch.int32, device="cuda"))
    B.kv_write(x, x, c, whole)
    q = _randn(g, 3 * rows, hq, hd, dtype=torch.bfloat16)
    say(f"[gpu] rows that see nothing, pages outside {kind} {rows}")
    on = B.KVBatch(table.cuda(), start.cuda(), kv_len.cuda())
    out, lse = B.kv_attn(q, c, on)
    pos = torch.cat([kv_len[s] - rows + torch.arange(rows) for s in range(3)])
    seq = torch.arange(3).repeat_interleave(rows)
    empty, bad = pos < 0, ((seq == 1) & (pos >= 32)) | ((seq == 2) & (pos >= 640))
    fine = ~empty & ~bad
    o, l = out.cpu(), lse.cpu()
    assert bool((o[empty] == 0).all()) and bool((l[:, empty] == -INF).all())
    assert o[bad].isnan().all() and l[:, bad].isnan().all()
    assert o[fine].isfinite().all() and l[:, fine].isfinite().all()
    # a window that has left the missing page behind
    out, lse = B.kv_attn(q, c, on, window=4, sinks=2)
    bad = ((seq == 1) & (pos >= 32) & (pos < 51)) | ((seq == 2) & (pos >= 640))
    assert out.cpu()[bad].isnan().all() and out.cpu()[~bad].isfinite().all()


@pytest.mark.parametrize("rows", [1, 5, 9, 40])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
@pytest.mark.parametrize("hd", [64, 128])
def test_what_a_missing_page_is_replaced_by_reaches_nobody(B, hd, kind, rows):
    """Pages that are no sequence's hold NaN; a row before the missing page, or
    behind it with a window, is what it is with the page there."""
    g = _gen(rows + hd)
    hq, hk, page = 8, 2, 16
    c = _cache(B, 20, page, hk, hd, kind)            # all NaN
    table = torch.arange(1, 20, dtype=torch.int32)[None].contiguous().cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    x = _randn(g, 200, hk, hd, dtype=torch.bfloat16)
    B.kv_write(x, x, c, B.KVBatch(table, i32(0, 200), i32(200)))
    broken = table.clone()
    broken[0, 5] = 77                                # positions 80 .. 95
    say(f"[gpu] a missing page {kind} {hd} {rows}")
    for last in (78 + rows, 83, 95, 100, 119, 160):
        q = _randn(g, rows, hq, hd, dtype=torch.bfloat16)
        pos = last - rows + torch.arange(rows)
        for window, sinks in ((0, 0), (20, 4), (20, 83)):
            want = B.kv_attn(q, c, B.KVBatch(table, i32(0, rows), i32(last)), window=window, sinks=sinks)
            got = B.kv_attn(q, c, B.KVBatch(broken, i32(0, rows), i32(last)), window=window, sinks=sinks)
            bad = (pos >= 80) & ((pos < 95 + window) | (window == 0) | (sinks > 80))
            assert want[0].isfinite().all() and got[0][bad].isnan().all() and got[1][:, bad].isnan().all()
            assert torch.equal(got[0][~bad], want[0][~bad]) and torch.equal(got[1][:, ~bad], want[1][:, ~bad]), (last, window, sinks)


def test_attention_strides_and_optional_outputs(B):
    g = _gen(8)
    batch = S.Batch([1, 20], [40, 3], 16, lead=1, trail=1)
    c = B.KVCache(*(_randn(g, batch.n_pages, 2, 16, 128, dtype=torch.float16) for _ in "kv"))
    on, rows = batch.device(B), batch.n
    q = _randn(g, rows, 4, 128, dtype=torch.float16)
    want, _ = B.kv_attn(q, c, on, out=torch.zeros_like(q))
    say("[gpu] attention strides")
    head_major = _randn(g, 4, rows, 128, dtype=torch.float16).transpose(0, 1)
    head_major.copy_(q)
    out = torch.zeros(rows, 4 * 128 + 8, device="cuda", dtype=torch.float16)[:, 8:].unflatten(1, (4, 128))
    B.kv_attn(head_major, c, on, out=out)
    assert torch.equal(out, want)
    one = q[:, :1].expand(rows, 4, 128)              # one head for all
    got, _ = B.kv_attn(one, c, on, out=torch.zeros_like(q))
    ref, _ = B.kv_attn(one.contiguous(), c, on, out=torch.zeros_like(q))
    assert torch.equal(got, ref)
    # the C entry without lse
    import ctypes as C
    args = B.pard_kv_attn_args(C.pointer(c.c), C.pointer(on.c(rows)), 4, B.PARD_F16, 0, 0, 128 ** -0.5)
    n = B.lib.pard_kv_attn_workspace_bytes(args)
    ws, out = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros_like(q)
    h = lambda t: B.pard_heads(t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
    assert B.lib.pard_kv_attn(args, h(q), h(out), None, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream) == B.PARD_OK
    assert torch.equal(out, want)
    empty, _ = B.kv_attn(q[:0], c, B.KVBatch(on.page_table, torch.zeros(3, dtype=torch.int32, device="cuda"), on.kv_len))
    assert empty.shape == (0, 4, 128)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_places_past_32_bits(B, kind):
    """Caches of more than 4 GiB, the sequences in their last pages."""
    hk, hd, page, size = 8, 128, 256, 2 if kind == "bf16" else 1
    n_pages = (5 << 30) // (hk * hd * page * size)
    g = _gen(3)
    say(f"[gpu] {n_pages} pages, {n_pages * hk * hd * page * size >> 20} MiB each {kind}")
    c = B.kv_cache(n_pages, page, hk, hd, T.DTYPES.get(kind, kind))
    for rows, past in (([1, 9], [300, 700]), ([200], [400])):
        batch = S.Batch(rows, past, page, spare=0)
        batch.table = np.where((batch.table >= 0) & (batch.table < batch.n_pages), n_pages - 1 - batch.table, -1).astype(np.int32)
        whole = S.Batch([r + p for r, p in zip(rows, past)], [0] * len(rows), page)
        whole.table = batch.table
        k, v = (_randn(g, whole.n, hk, hd, dtype=torch.bfloat16) for _ in "kv")
        on = whole.device(B)
        B.kv_write(k, v, c, on)
        held = [S.stored(x, kind) if kind in S.BITS else x.double().cpu() for x in (k, v)]
        for got, want in zip(B.kv_read(c, on, whole.n), held):
            assert torch.equal(got.double().cpu(), want)
        q = _randn(g, batch.n, 16, hd, dtype=torch.bfloat16)
        out, lse = B.kv_attn(q, c, batch.device(B))
        at = lambda x: lambda s, j: x[int(whole.row_start[s]) + torch.as_tensor(j)]  # noqa: E731
        ref = S.attn_ref(q, at(held[0]), at(held[1]), batch, hd ** -0.5)
        T.assert_within(out, *ref["out"], "out")
        T.assert_within(lse, *ref["lse"], "lse")
    del c
    torch.cuda.empty_cache()


# --------------------------------------------------------------------------
# logits
# --------------------------------------------------------------------------

LOGITS = [(1, 1, 1, 5), (4, 3, 70, 20), (9, 1, 2048, 40), (12, 4, 2049, 0), (33, 5, 4097, 300), (2, 2, 33, 1), (40, 40, 999, 9), (3, 1, 8191, 2000)]


def _logits_case(g, rows, seqs, vocab, history, dt):
    randint = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    rand = lambda n: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    logits = _randn(g, rows, vocab + 3, dtype=dt, std=3.0)[:, :vocab]
    # few ids often, some outside the vocabulary
    tokens = (rand(seqs * max(history, 1)) ** 3 * (vocab + 2)).to(torch.int32).view(seqs, -1) - 1
    row_seq = torch.arange(rows, dtype=torch.int32, device="cuda") * seqs // rows
    row_len = randint(-2, history + 5, rows)
    if rows > 5:
        row_len[:5] = torch.arange(5, device="cuda")  # a history that grows
        row_seq[:5] = 0
        row_seq[5] = -1
    count = np.arange(seqs) % 3 * 4
    start = torch.from_numpy(np.concatenate([[0], np.cumsum(count)])).to(torch.int32).cuda()
    n = int(count.sum())
    ids = randint(-1, vocab + 1, n)
    if n > 3:
        ids[1] = ids[3]                              # an id twice in a list
    masks = randint(-(1 << 31), (1 << 31) - 1, rows + 1, (vocab + 31) // 32)
    mask_row = randint(-1, rows + 2, rows)
    masks[0] = 0                                     # a state that allows nothing
    mask_row[0] = 0
    return logits, dict(tokens=tokens, row_len=row_len, prompt_len=randint(-1, history + 2, seqs), row_seq=row_seq), dict(
        repetition=1 + rand(seqs), presence=rand(seqs) - 0.3, frequency=rand(seqs) - 0.3, bias=(start, ids, 4 * _randn(g, n)),
        mask=masks, mask_row=mask_row)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", LOGITS, ids=str)
def test_logits(B, shape, dtype):
    rows, seqs, vocab, history = shape
    g, dt = _gen(vocab + rows), T.DTYPES[dtype]
    logits, base, steps = _logits_case(g, rows, seqs, vocab, history, dt)
    say(f"[gpu] logits {shape} {dtype}")
    cpu = lambda d: {k: tuple(t.cpu() for t in v) if isinstance(v, tuple) else v.cpu() for k, v in d.items()}  # noqa: E731
    for names in (list(steps), ["repetition"], ["frequency", "presence"], ["bias"], ["mask", "mask_row"], []):
        some = {k: steps[k] for k in names}
        out, best = B.logits_adjust(logits, **base, **some)
        c = cpu(base) | cpu(some)
        if "mask" in c:
            c["mask"] = c["mask"].numpy().astype(np.int64) & 0xffffffff
        want, bound = S.logits_ref(logits, **c)
        hidden = torch.isinf(want)
        assert torch.equal(torch.isinf(out.cpu()), hidden)
        T.assert_within(out.masked_fill(hidden.cuda(), 0.0), want.masked_fill(hidden, 0.0), bound, f"{names}")
        assert best.tolist() == S.best_of(out)
    # in place, and without the pick
    same = logits.clone()
    got, none = B.logits_adjust(same, **base, **steps, out=same, best=False)
    assert got is same and none is None and torch.equal(same, B.logits_adjust(logits, **base, **steps)[0])
    # strides that no 16-byte access fits
    odd = torch.empty(rows, vocab + 1, device="cuda", dtype=dt)[:, 1:].copy_(logits)
    got = B.logits_adjust(odd, **base, **steps)
    want = B.logits_adjust(logits, **base, **steps)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_logits_special_values(B):
    x = torch.tensor([[NAN, 1.0, 1.0, -INF], [-INF] * 4, [NAN] * 4, [-0.0, 0.0, -1.0, -0.0], [INF, INF, 3.0, NAN]], device="cuda")
    assert B.logits_adjust(x)[1].tolist() == [1, -1, -1, 0, 0]
    lens = torch.full((5,), 4, dtype=torch.int32, device="cuda")
    tokens = torch.tensor([[0, 1, 2, 3]] * 5, dtype=torch.int32, device="cuda")
    two = torch.full((5,), 2.0, device="cuda")
    y, best = B.logits_adjust(x, tokens, lens, repetition=two, frequency=two)
    want = torch.tensor([[NAN, -1.5, -1.5, -INF], [-INF] * 4, [NAN] * 4, [-2.0, -2.0, -4.0, -2.0], [INF, INF, -0.5, NAN]])
    assert torch.equal(y.cpu().nan_to_num(99.0), want.nan_to_num(99.0)) and best.tolist() == [1, -1, -1, 0, 0]
    # rows that a mask leaves nothing of, of NaN too; a mask row that is not there
    mask = torch.tensor([[0], [8]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, -1, 0, 1, 2], dtype=torch.int32, device="cuda")
    y, best = B.logits_adjust(x, mask=mask, mask_row=rows)
    assert best.tolist() == [-1, -1, -1, 3, -1] and bool((y[[0, 2, 4]] == -INF).all()) and y[3].tolist() == [-INF, -INF, -INF, 0.0]
    y, best = B.logits_adjust(x[:0])
    assert y.shape == (0, 4) and best.shape == (0,)


def test_logits_large(B):
    """A real vocabulary, rows that share a growing history."""
    g = _gen(0)
    vocab, rows = 128256, 27
    logits = _randn(g, rows, vocab)
    tokens = torch.randint(0, vocab, (3, 5000), generator=g, device="cuda", dtype=torch.int32)
    tokens[0] = 77                                   # one token, over and over
    seq = torch.arange(3, dtype=torch.int32, device="cuda").repeat_interleave(9)
    lens = 4900 + torch.arange(9, dtype=torch.int32, device="cuda").repeat(3)
    three = torch.full((3,), 0.01, device="cuda")
    say("[gpu] logits large")
    y, best = B.logits_adjust(logits, tokens, lens, row_seq=seq, frequency=three)
    want = logits.double()
    want[:9, 77] -= 0.01 * lens[:9].double()
    for r in range(9, 27):
        want[r] -= 0.01 * torch.bincount(tokens[int(seq[r]), :int(lens[r])].long(), minlength=vocab).double()
    assert bool(((y.double() - want).abs() <= 4 * T.F * (want.abs() + 50)).all()) and best.tolist() == S.best_of(y)


# --------------------------------------------------------------------------
# streams, graphs, and all of them together
# --------------------------------------------------------------------------

class _Step:
    """The new rows of a batch through two layers of a decoder: norms and
    projections by torch, rotation, cache, attention and logits by the library."""

    def __init__(self, B, g, kind, hq=8, hk=2, hd=64, d=128, vocab=500, page=16, n_pages=64):
        self.B, self.hq, self.hk, self.hd, self.vocab, self.page = B, hq, hk, hd, vocab, page
        w = lambda *s: _randn(g, *s, dtype=torch.bfloat16, std=s[0] ** -0.5)  # noqa: E731
        self.embed = _randn(g, vocab, d, dtype=torch.bfloat16)
        self.layers = [dict(qkv=w(d, (hq + 2 * hk) * hd), o=w(hq * hd, d)) for _ in range(2)]
        self.head = w(d, vocab)
        self.caches = [_cache(B, n_pages, page, hk, hd, kind) for _ in self.layers]
        self.table = B.rope_table(256, hd, 1e4)

    def __call__(self, ids, positions, on, adjust):
        B, hq, hk, hd = self.B, self.hq, self.hk, self.hd
        x = self.embed[ids]
        for layer, cache in zip(self.layers, self.caches):
            n = torch.nn.functional.rms_norm(x.float(), x.shape[1:]).to(x.dtype)
            qkv = n @ layer["qkv"]
            q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([hq * hd, hk * hd, hk * hd], 1))
            q, k = B.qk_rope(q, k, positions, self.table)
            B.kv_write(k, v, cache, on)
            out, _ = B.kv_attn(q, cache, on)
            x = x + out.flatten(1) @ layer["o"]
        n = torch.nn.functional.rms_norm(x.float(), x.shape[1:]).to(x.dtype)
        return B.logits_adjust((n @ self.head).float(), **adjust)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_step_at_once_is_its_tokens_one_by_one(B, kind):
    """Prompts in one pass and a verify pass of K + 1 rows give the logits of
    passes of single tokens (attention of different splits: bf16 roundings apart),
    and the same picks where they are clear; rollback is a smaller length."""
    g = _gen(5)
    step, rng = _Step(B, g, kind), np.random.default_rng(0)
    other = _Step(B, _gen(5), kind)
    lens, k = [5, 21, 40], 6
    ids = [rng.integers(0, 500, n + k) for n in lens]
    table = torch.from_numpy(rng.permutation(64)[:3 * 8].reshape(3, 8).astype(np.int32)).cuda()
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    tokens = i32([np.pad(t, (0, 64 - len(t))) for t in ids])
    penalties = dict(repetition=torch.full((3,), 1.3, device="cuda"), frequency=torch.full((3,), 0.1, device="cuda"),
                     prompt_len=i32(lens))

    def run(m, first, last):
        """The rows first[s] .. last[s] - 1 of every sequence."""
        n = [b - a for a, b in zip(first, last)]
        pos = np.concatenate([np.arange(a, b) for a, b in zip(first, last)])
        on = B.KVBatch(table, i32(np.concatenate([[0], np.cumsum(n)])), i32(last))
        at = torch.from_numpy(np.concatenate([t[a:b] for t, a, b in zip(ids, first, last)])).cuda()
        seq = i32(np.repeat(np.arange(3), n))
        return m(at, i32(pos), on, dict(tokens=tokens, row_len=i32(pos + 1), row_seq=seq, **penalties))
    say(f"[gpu] steps {kind}")
    run(step, [0, 0, 0], lens)
    wrong = [n + 3 for n in lens]
    run(step, lens, wrong)                           # candidates that are not kept: the next pass overwrites them
    got, best = run(step, lens, [n + k for n in lens])
    rows = [[], [], []]
    for i in range(max(lens) + k):
        first = [min(i, n + k) for n in lens]
        last = [min(i + 1, n + k) for n in lens]
        y, b = run(other, first, last)
        at = 0
        for s in range(3):
            if last[s] > first[s]:
                if i >= lens[s]:
                    rows[s].append((y[at], int(b[at])))
                at += 1
    for i, (y, b) in enumerate(r for s in rows for r in s):
        assert bool(((got[i] - y).abs() <= 0.08).all()), f"row {i}: {float((got[i] - y).abs().max())}"
        top = y.topk(2).values
        if float(top[0] - top[1]) > 0.16:
            assert int(best[i]) == b


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_captured_calls_follow_what_changes(B, kind):
    """A graph of cache, attention and logits, replayed beside eager work after the
    tables, lengths, rows and tokens have changed, every replay against the eager
    result; another graph beside it has its own workspace."""
    g = _gen(6)
    hq, hk, hd, page = 8, 2, 64, 16
    def state(rows, past, seed):
        b = S.Batch(rows, past, page, seed=seed)
        table = np.full((3, 40), -1, np.int32)
        table[:, :b.width] = b.table
        return [torch.from_numpy(x).cuda() for x in (table, b.row_start, b.kv_len)]
    states = [state([1, 9, 3], [300, 20, 600], 1), state([4, 1, 8], [10, 500, 0], 2), state([0, 13, 0], [3, 200, 5], 3)]
    c = _cache(B, 140, page, hk, hd, kind)
    for t in (c.k, c.v):
        t.copy_(torch.randint(0, 16, t.shape, generator=g, device="cuda").to(t.dtype))
    if c.k_scale is not None:
        c.k_scale.fill_(126), c.v_scale.fill_(127)
    rows = 13
    now = [t.clone() for t in states[0]]
    q, k, v = (_randn(g, rows, h, hd, dtype=torch.bfloat16) for h in (hq, hk, hk))
    logits, tokens = _randn(g, rows, 3001), torch.randint(0, 3001, (rows, 50), generator=g, device="cuda", dtype=torch.int32)
    lens, one = torch.randint(0, 50, (rows,), generator=g, device="cuda", dtype=torch.int32), torch.ones(rows, device="cuda")

    def chain(on):
        B.kv_write(k, v, c, on)
        out, lse = B.kv_attn(q, c, on)
        small, _ = B.kv_attn(q, c, on, window=33, sinks=2)
        back = B.kv_read(c, on, rows)
        y, best = B.logits_adjust(logits, tokens, lens, presence=one)
        return out, lse, small, *back, y, best
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for _ in range(2):
        on = B.KVBatch(*now)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            chain(on)
        torch.cuda.current_stream().wait_stream(side)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(chain(on))
        graphs.append(gr)
    for turn in range(6):
        say(f"[gpu] replay {turn} {kind}")
        for t, new in zip(now, states[turn % 3]):
            t.copy_(new)
        q.copy_(_randn(g, *q.shape, dtype=q.dtype))
        k.copy_(_randn(g, *k.shape, dtype=q.dtype))
        logits.normal_(generator=g)
        lens.copy_(torch.randint(0, 50, (rows,), generator=g, device="cuda", dtype=torch.int32))
        n = int(now[1][-1])
        want = [t.clone() for t in chain(B.KVBatch(*now))]
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        if turn == 4:                                # both at once, on two streams
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graphs[1].replay()
            torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for got in outs if turn == 4 else [outs[turn % 2]]:
            for i, (a, w) in enumerate(zip(got, want)):
                a, w = (a[:, :n], w[:, :n]) if i == 1 else (a, w) if i > 4 else (a[:n], w[:n])
                assert torch.equal(a, w), (turn, i)


def test_streams(B):
    """Calls on a side stream with inputs made there, and the stream's tensors reused."""
    g = _gen(7)
    batch = S.Batch([1, 30], [50, 9], 16)
    c = B.KVCache(*(_randn(g, batch.n_pages, 2, 16, 64, dtype=torch.bfloat16) for _ in "kv"))
    q, on = _randn(g, batch.n, 4, 64, dtype=torch.bfloat16), batch.device(B)
    k = _randn(g, batch.n, 2, 64, dtype=torch.bfloat16)
    logits = _randn(g, 4, 50000)
    B.kv_write(k, k, c, on)
    want = [t.clone() for t in (*B.kv_attn(q, c, on), *B.kv_read(c, on, batch.n), *B.logits_adjust(logits))]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(3):
        st.wait_stream(torch.cuda.current_stream())
        a, b, d = q.clone(), k.clone(), logits.clone()
        st.wait_stream(torch.cuda.current_stream())
        B.kv_write(b, b, c, on, stream=st)
        got = (*B.kv_attn(a, c, on, stream=st), *B.kv_read(c, on, batch.n, stream=st), *B.logits_adjust(d, stream=st))
        del a, b, d
        junk = [torch.full_like(t, 3) for t in (q, k, logits)]
        torch.cuda.current_stream().wait_stream(st)
        torch.cuda.synchronize()
        for x, w in zip(got, want):
            assert torch.equal(x, w)
        del junk


def test_binding_refuses(B):
    g = _gen(9)
    batch = S.Batch([2], [3], 16)
    c, on = _cache(B, batch.n_pages, 16, 2, 64, "e4m3"), batch.device(B)
    q, k = _randn(g, 2, 4, 64, dtype=torch.bfloat16), _randn(g, 2, 2, 64, dtype=torch.bfloat16)
    x = _randn(g, 2, 64)
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    for f, word in ((lambda: B.kv_attn(_randn(g, 2, 4, 128, dtype=torch.bfloat16), c, on), "head_dim"), (lambda: B.kv_attn(q.float(), c, on), "pard_kv_attn"),
                    (lambda: B.kv_attn(q, c, on, out=q), "pard_kv_attn"), (lambda: B.kv_attn(q[:, :3], c, on), "pard_kv_attn"),
                    (lambda: B.kv_write(q, q, c, on), "shape"), (lambda: B.kv_write(k, k[:1], c, on), "shape"),
                    (lambda: B.kv_read(c, on, 2, torch.int32), "dtype"), (lambda: B.kv_read(c, on, 2, k_out=k, v_out=k), "pard_kv_read"),
                    (lambda: B.KVCache(c.k, c.v), "without scales"), (lambda: B.KVCache(c.k, c.v, c.k_scale), "one form"),
                    (lambda: B.KVCache(c.k, c.v, c.k_scale, c.v_scale[..., :1].contiguous()), "scales"),
                    (lambda: B.KVBatch(on.page_table, on.row_start, on.kv_len.long()), "kv_len"),
                    (lambda: B.logits_adjust(x, tokens=i[None]), "row_len"), (lambda: B.logits_adjust(x, repetition=x[0, :2].contiguous()), "pard_logits_adjust"),
                    (lambda: B.logits_adjust(x, mask=i[:, None]), "mask"), (lambda: B.logits_adjust(x, out=x[:1]), "out")):
        with pytest.raises(B.PardError, match=word):
            f()
