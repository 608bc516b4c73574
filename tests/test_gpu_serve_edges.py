"""GPU checks of the serving operators at the ends of what their documentation allows:
lengths past the page table beside windows and first tokens, every scale byte of a
cache, float16 over long contexts, the documented order of the logits' operations, empty
histories, masks and biases, windows past 32 bits."""
import numpy as np
import pytest
import torch

import serve_bounds as SB
import serve_common as S
import test_gpu_serve as G
import train_common as T
from gpu_common import say
from test_gpu_serve import B, INF, _gen, _randn  # noqa: F401

pytestmark = pytest.mark.gpu


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# --------------------------------------------------------------------------
# lengths past the table
# --------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 5, 9, 40, 150])
@pytest.mark.parametrize("kind", ["bf16", "e4m3", "e2m1"])
def test_a_window_past_the_table_beside_more_first_tokens_than_it_names(B, kind, rows):  # noqa: F811
    """The last sequence's rows past its table are NaN; the others are what they are
    by themselves."""
    g = _gen(rows)
    hq, hk, hd, page, pages = 8, 2, 64, 16, 64
    c = G._cache(B, 2 * pages, page, hk, hd, kind)
    table = torch.arange(2 * pages, dtype=torch.int32, device="cuda").view(2, pages)
    x = _randn(g, 2 * pages * page, hk, hd, dtype=torch.bfloat16)
    B.kv_write(x, x, c, B.KVBatch(table, _i32(0, 1024, 2048), _i32(1024, 1024)))
    q = _randn(g, 2 * rows, hq, hd, dtype=torch.bfloat16)
    for window, sinks in ((100, 2048), (100, 1025), (1, 1 << 30), (100, 4), (1024, 2048)):
        for past in (2200, 1023 + rows, 1024 + rows + 100, 1024 + rows // 2):
            say(f"[gpu] past the table {kind} {rows} {window} {sinks} {past}")
            out, lse = B.kv_attn(q, c, B.KVBatch(table, _i32(0, rows, 2 * rows), _i32(900, past)), window=window, sinks=sinks)
            one, one_lse = B.kv_attn(q[:rows], c, B.KVBatch(table[:1].contiguous(), _i32(0, rows), _i32(900)), window=window, sinks=sinks)
            T.assert_within(out[:rows], one.double().cpu(), 2.0 ** -6 * one.double().cpu().abs() + 2.0 ** -6, "the other sequence")
            bad = torch.cat([torch.zeros(rows, dtype=torch.bool), past - rows + torch.arange(rows) >= 1024])
            assert out.cpu()[bad].isnan().all() and lse.cpu()[:, bad].isnan().all()
            assert out.cpu()[~bad].isfinite().all() and lse.cpu()[:, ~bad].isfinite().all()


# --------------------------------------------------------------------------
# float16
# --------------------------------------------------------------------------

LONG = [([1], [4000], 4096, 4, 1, 128), ([13, 2], [900, 1500], 128, 28, 4, 128), ([9], [9000], 16, 16, 4, 64), ([1], [20000], 64, 8, 1, 128),
        ([70], [8000], 16, 4, 2, 64), ([2, 5], [12000, 30], 32, 16, 2, 64), ([9, 9], [9000, 200], 16, 8, 2, 128)]


@pytest.mark.parametrize("kind", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: f"{s[0]}-{s[1]}-{s[2:]}")
def test_float16_over_long_contexts(B, monkeypatch, shape, kind):  # noqa: F811
    monkeypatch.setattr(S, "attn_ref", SB.sharp_attn_ref)
    G._check_attn(B, *shape, "f16", kind, lead=1, trail=2)


@pytest.mark.parametrize("shape", G.ATTN, ids=lambda s: f"{s[0][:3]}-{s[1][:3]}-{s[2:]}")
def test_float16(B, monkeypatch, shape):  # noqa: F811
    monkeypatch.setattr(S, "attn_ref", SB.sharp_attn_ref)
    for kind in ("f16", "e4m3", "e2m1"):
        G._check_attn(B, *shape, "f16", kind)


@pytest.mark.parametrize("kind", ["f16", "e4m3", "e2m1"])
def test_float16_peaked_and_within_windows(B, monkeypatch, kind):  # noqa: F811
    """Probabilities far below the largest, which float16 holds as subnormals."""
    monkeypatch.setattr(S, "attn_ref", SB.sharp_attn_ref)
    for window, sinks, std in ((0, 0, 3.0), (0, 0, 8.0), (500, 4, 3.0), (100, 300, 2.0)):
        G._check_attn(B, [1, 9, 2], [3000, 600, 40], 16, 8, 2, 64, "f16", kind, window, sinks, std=std)
        G._check_attn(B, [5, 150], [1200, 70], 32, 8, 2, 128, "f16", kind, window, sinks, std=std)


# --------------------------------------------------------------------------
# every scale byte
# --------------------------------------------------------------------------

def _bytes(g, *shape):
    return torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_reading_every_scale_byte(B, kind):  # noqa: F811
    """All codes under the scales 2^-127 to 2^127 and NaN, rounded once to each type."""
    for hd in (64, 128):
        g = _gen(hd)
        c = G._cache(B, 64, 16, 1, hd, kind)
        for t in (c.k, c.v):
            t.copy_(_bytes(g, *t.shape))
        n = 64 * 16
        c.k_scale.copy_((torch.arange(n * hd // 32, device="cuda") % 256).to(torch.uint8).view(c.k_scale.shape))
        c.v_scale.copy_(_bytes(g, *c.v_scale.shape))
        on = B.KVBatch(torch.arange(64, dtype=torch.int32, device="cuda")[None].contiguous(), _i32(0, n), _i32(n))
        for dtype in ("f32", "bf16", "f16"):
            say(f"[gpu] scale bytes {kind} {hd} {dtype}")
            for got, t, s in zip(B.kv_read(c, on, n, T.DTYPES[dtype]), (c.k, c.v), (c.k_scale, c.v_scale)):
                # (a value has 4 bits at most: float32 holds all within its range, and loses what is below)
                want = S.decoded(t, s, kind).view(n, 1, hd).float().to(T.DTYPES[dtype])
                nan = want.isnan()
                assert torch.equal(got.cpu().isnan(), nan)
                off = (got.cpu() != want) & ~nan
                assert not bool(off.any()), (int(off.sum()), got.cpu()[off][:4], want[off][:4], s.view(n, -1).cpu()[off.nonzero()[:4, 0]])


@pytest.mark.parametrize("rows", [1, 5, 9, 40, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_attention_over_every_scale(B, kind, dtype, rows):  # noqa: F811
    """Keys and values whose blocks have scales from 2^-127 on; and, in a sequence of
    their own, blocks of NaN."""
    dt = T.DTYPES[dtype]
    for hd in (64, 128):
        g = _gen(rows + hd)
        hq, hk, page, n = 8, 2, 16, 320
        c = G._cache(B, 41, page, hk, hd, kind)
        for t in (c.k, c.v):
            # (no codes of NaN)
            t.copy_(_bytes(g, *t.shape) & 0xf7 if kind == "e4m3" else _bytes(g, *t.shape))
        small = torch.tensor([0, 1, 2, 60, 110, 112, 114, 119, 120, 121], dtype=torch.uint8, device="cuda")
        for t in (c.k_scale, c.v_scale):
            t.copy_(small[torch.randint(0, len(small), t.shape, generator=g, device="cuda")])
        q = _randn(g, 2 * rows, hq, hd, dtype=dt, std=0.25)
        table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
        on = B.KVBatch(table, _i32(0, rows, 2 * rows), _i32(n, n))
        say(f"[gpu] attention over every scale {kind} {dtype} {hd} {rows}")
        batch = S.Batch([rows, rows], [n - rows] * 2, page)

        def of(t, s):
            v = S.decoded(t, s, kind)[:40].transpose(1, 2).reshape(2, n, hk, hd).to(torch.float32).to(dt).double()
            return lambda seq, j: v[seq, torch.as_tensor(j)]
        ref = SB.sharp_attn_ref(q, of(c.k, c.k_scale), of(c.v, c.v_scale), batch, hd ** -0.5)
        out, lse = B.kv_attn(q, c, on)
        # (2^-118: what products of the smallest values lose below float32's normal range)
        T.assert_within(out, ref["out"][0], ref["out"][1] + 2.0 ** -118, "out")
        T.assert_within(lse, *ref["lse"], "lse")
        # one key, then one value, of the second sequence NaN: key head 1, position 3
        for t in (c.k_scale, c.v_scale):
            old = t[20, 1, 3, 0].clone()
            t[20, 1, 3, 0] = 255
            got, got_lse = B.kv_attn(q, c, on)
            assert torch.equal(got[:rows], out[:rows]) and torch.equal(got_lse[:, :rows], lse[:, :rows])
            assert torch.equal(got[rows:, :4], out[rows:, :4])           # heads of key head 0
            bad = got[rows:, 4:] if t is c.k_scale else got[rows:, 4:, :32]
            assert bad.isnan().all()
            t[20, 1, 3, 0] = old


# --------------------------------------------------------------------------
# windows and hints past 32 bits
# --------------------------------------------------------------------------

def test_sizes_past_32_bits(B):  # noqa: F811
    """A window, first tokens or a hint of 2^32 and a few are large, not a few."""
    g = _gen(3)
    batch = S.Batch([1, 20], [300, 90], 16)
    c = B.KVCache(*(_randn(g, batch.n_pages, 2, 16, 64, dtype=torch.bfloat16) for _ in "kv"))
    q, on = _randn(g, batch.n, 4, 64, dtype=torch.bfloat16), batch.device(B)
    say("[gpu] windows past 32 bits")
    want, want_lse = B.kv_attn(q, c, on)
    for size in (2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, 2 ** 70):
        for kw in (dict(window=size), dict(window=7, sinks=size)):
            out, lse = B.kv_attn(q, c, on, **kw)
            assert torch.equal(out, want) and torch.equal(lse, want_lse), (size, kw)
        far = batch.device(B, size)
        assert far.max_seq_rows > 0
        out, _ = B.kv_attn(q, c, far)
        T.assert_within(out, want.double().cpu(), 2.0 ** -6 * want.double().cpu().abs() + 2.0 ** -7, "hint")
    for kw in (dict(window=-1), dict(window=-2 ** 32), dict(window=-2 ** 40 + 3), dict(window=7, sinks=-2 ** 32 + 1)):
        with pytest.raises(B.PardError, match="pard_kv_attn"):
            B.kv_attn(q, c, on, **kw)
    with pytest.raises(B.PardError, match="pard_kv_attn"):
        B.kv_attn(q, c, batch.device(B, -2 ** 32 + 1))


# --------------------------------------------------------------------------
# logits
# --------------------------------------------------------------------------

def _in_order(x, tokens, row_len, prompt_len, row_seq, repetition, presence, frequency, bias):
    """The documented steps as single float32 operations, one after the other."""
    y, vocab = x.float().cpu().numpy().copy(), x.shape[1]
    f32 = np.float32
    for r in range(len(y)):
        s = int(row_seq[r])
        h = tokens[s, :int(row_len[r])].numpy()
        had = np.bincount(h, minlength=vocab)[:vocab] > 0
        c = np.bincount(h[int(prompt_len[s]):], minlength=vocab)[:vocab]
        rep, pre, fre = (f32(t[s]) for t in (repetition, presence, frequency))
        y[r] = np.where(had, np.where(y[r] > 0, y[r] / rep, y[r] * rep), y[r])
        step = fre * c.astype(f32)
        y[r] = np.where(c > 0, y[r] - step, y[r])
        y[r] = np.where(c > 0, y[r] - pre, y[r])
        lo, hi = int(bias[0][s]), int(bias[0][s + 1])
        for t, b in {int(t): f32(b) for t, b in zip(bias[1][lo:hi], bias[2][lo:hi])}.items():
            y[r, t] = y[r, t] + b
    return torch.from_numpy(y).to(x.dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [70, 4096, 9001])
def test_logits_are_the_documented_operations(B, dtype, vocab):  # noqa: F811
    """Bit by bit: no product and sum become one operation."""
    g = _gen(vocab)
    rows, seqs, history = 24, 4, 3000
    logits = _randn(g, rows, vocab, dtype=T.DTYPES[dtype], std=4.0)
    tokens = torch.randint(0, vocab, (seqs, history), generator=g, device="cuda", dtype=torch.int32)
    rand = lambda n: torch.rand(n, generator=g, device="cuda")  # noqa: E731
    row_seq = torch.arange(rows, dtype=torch.int32, device="cuda") * seqs // rows
    row_len = history - rows + torch.arange(rows, dtype=torch.int32, device="cuda")
    args = dict(tokens=tokens, row_len=row_len, prompt_len=_i32(0, 700, 10, 2999), row_seq=row_seq, repetition=1 + rand(seqs),
                presence=rand(seqs) - 0.3, frequency=rand(seqs) / 3,
                bias=(_i32(0, 40, 40, 60, 60), torch.randint(0, vocab, (60,), generator=g, device="cuda", dtype=torch.int32), _randn(g, 60)))
    say(f"[gpu] logits in order {dtype} {vocab}")
    out, best = B.logits_adjust(logits, **args)
    want = _in_order(logits, **{k: tuple(t.cpu() for t in v) if isinstance(v, tuple) else v.cpu() for k, v in args.items()})
    off = out.cpu() != want
    assert not bool(off.any()), f"{int(off.sum())} of {off.numel()} differ, first {out.cpu()[off][:3].tolist()} for {want[off][:3].tolist()}"
    assert best.tolist() == S.best_of(want)


def test_empty_histories(B):  # noqa: F811
    """Sequences without a token yet: penalties change nothing."""
    x = _randn(_gen(1), 3, 700)
    none, lens, one = torch.empty(3, 0, dtype=torch.int32, device="cuda"), _i32(0, 5, -1), torch.full((3,), 1.5, device="cuda")
    say("[gpu] empty histories")
    for kw in (dict(repetition=one), dict(presence=one), dict(frequency=one), dict(repetition=one, presence=one, frequency=one), {}):
        out, best = B.logits_adjust(x, none, lens, **kw)
        assert torch.equal(out, x) and best.tolist() == S.best_of(x)


def test_masks_of_no_rows(B):  # noqa: F811
    """A row's mask that is not there allows nothing, also where none is."""
    x = _randn(_gen(2), 4, 70)
    mask = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    say("[gpu] masks of no rows")
    out, best = B.logits_adjust(x, mask=mask, mask_row=_i32(0, -1, 7, -5))
    assert bool((out[[0, 2]] == -INF).all()) and torch.equal(out[[1, 3]], x[[1, 3]])
    assert best.tolist() == [-1, int(x[1].argmax()), -1, int(x[3].argmax())]


def test_biases_of_no_sequences(B):  # noqa: F811
    """bias starts of one entry are those of no sequence: nothing behind it is read."""
    x = _randn(_gen(3), 1, 70)
    say("[gpu] biases of no sequences")
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")[:1]
    out, best = B.logits_adjust(x, bias=(start, _i32(5), torch.full((1,), 100.0, device="cuda")), row_seq=_i32(0))
    assert torch.equal(out, x) and best.tolist() == S.best_of(x)
