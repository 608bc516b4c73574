"""ctypes binding of libpard.so (include/pard.h): argument marshalling only.

Every computation runs in the HIP library; this module converts Python /
numpy / torch arguments to the C ABI and raises ``PardError`` on a non-OK
status.  PyTorch is used only to allocate the device arena and to name the
HIP stream.  Importing fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpard.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_18583_amd.csrc.build` "
                      "(or __graft_entry__.build())")

lib = C.CDLL(LIB_PATH)

PARD_OK, PARD_ERR_ARG, PARD_ERR_STATE, PARD_ERR_CAPACITY = 0, -1, -2, -3
PARD_ERR_NOMEM, PARD_ERR_DEVICE, PARD_ERR_UNSUPPORTED, PARD_ERR_RANGE = -4, -5, -6, -7
PARD_F32, PARD_BF16, PARD_F16 = 0, 1, 2
PARD_TARGET, PARD_DRAFT = 0, 1
PARD_MODE_PARALLEL, PARD_MODE_VANILLA = 0, 1
PARD_ROPE_PLAIN, PARD_ROPE_LINEAR, PARD_ROPE_LLAMA3, PARD_ROPE_YARN = range(4)
PARD_ROPE_HALF, PARD_ROPE_INTERLEAVED = 0, 1
OP_EMBED, OP_QKV, OP_ATTN, OP_O, OP_GATEUP, OP_DOWN, OP_LM, OP_TAIL = range(8)


class pard_model_spec(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn_dim", C.c_int32),
                ("vocab", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("init_std", C.c_float), ("qkv_bias", C.c_int32), ("tied_embeddings", C.c_int32),
                ("dtype", C.c_int32), ("weight_stream", C.c_uint32), ("seed", C.c_uint64),
                ("rope_factor", C.c_float), ("rope_low_freq_factor", C.c_float),
                ("rope_high_freq_factor", C.c_float), ("rope_original_max_pos", C.c_int32)]


class pard_stats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("tokens", C.c_int64), ("elapsed_ms", C.c_double),
                ("draft_ms", C.c_double), ("verify_ms", C.c_double), ("accept_ms", C.c_double),
                ("step_ms_p50", C.c_double), ("step_ms_p90", C.c_double),
                ("accept_hist", C.c_int64 * 33)]


class pard_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class pard_rope_spec(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32), ("theta", C.c_float), ("factor", C.c_float),
                ("low", C.c_float), ("high", C.c_float), ("original_max_pos", C.c_int32)]


class pard_rope_args(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n_q", C.c_int32), ("n_k", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("n_pos", C.c_int32),
                ("eps", C.c_float), ("positions", C.c_void_p), ("table", C.c_void_p), ("q_gain", C.c_void_p),
                ("k_gain", C.c_void_p)]


class pard_cod_plan(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n_samples", C.c_int32), ("n_tiles", C.c_int32), ("data", C.c_void_p)]


class pard_cod_attn_args(C.Structure):
    _fields_ = [("plan", C.POINTER(pard_cod_plan)), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float)]


class pard_cod_loss_args(C.Structure):
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int32), ("dtype", C.c_int32), ("n_sections", C.c_int32),
                ("grad_scale", C.c_float), ("logits", C.c_void_p), ("logits_stride", C.c_int64),
                ("labels", C.c_void_p), ("section", C.c_void_p), ("weights", C.POINTER(C.c_float)),
                ("d_logits", C.c_void_p), ("d_stride", C.c_int64), ("loss", C.c_void_p), ("row_loss", C.c_void_p)]


_I32P = C.POINTER(C.c_int32)
_HEADSP = C.POINTER(pard_heads)
_SPECP = C.POINTER(pard_model_spec)
_CTX = C.c_void_p

_sig = {
    "pard_arena_bytes": (C.c_size_t, [_SPECP, _SPECP, C.c_int32, C.c_int32, C.c_int32]),
    "pard_model_load": (C.c_int, [_SPECP, _SPECP, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(_CTX)]),
    "pard_prefill": (C.c_int, [_CTX, C.c_int32, _I32P, C.c_int32, _I32P]),
    "pard_draft": (C.c_int, [_CTX, C.c_int32, _I32P, C.c_int32, C.c_int32, _I32P]),
    "pard_verify": (C.c_int, [_CTX, C.c_int32, _I32P, C.c_int32, _I32P, _I32P]),
    "pard_kv_truncate": (C.c_int, [_CTX, C.c_int32, C.c_int32, C.c_int32]),
    "pard_kv_len": (C.c_int, [_CTX, C.c_int32, C.c_int32, _I32P]),
    "pard_generate": (C.c_int, [_CTX, C.c_int32, _I32P, C.c_int32, C.c_int32, C.c_int32, _I32P,
                                C.POINTER(pard_stats)]),
    "pard_generate_ex": (C.c_int, [_CTX, C.c_int32, _I32P, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                   _I32P, C.POINTER(pard_stats)]),
    "pard_set_sampling": (C.c_int, [_CTX, C.c_float, C.c_uint64]),
    "pard_cod_capacity": (C.c_int64, [C.c_int32, C.c_int32, C.c_double, C.c_double]),
    "pard_cod_layout": (C.c_int64, [C.POINTER(C.c_int64), C.c_int32, C.c_int32, C.c_double, C.c_double,
                                    C.POINTER(C.c_int64)]),
    "pard_cod_workspace_bytes": (C.c_size_t, [C.c_int32]),
    "pard_cod_build": (C.c_int, [C.c_void_p, C.POINTER(C.c_int64), C.c_int32, C.c_int32, C.c_double,
                                 C.c_double, C.c_int32, C.c_uint64, C.POINTER(C.c_int64), C.c_void_p,
                                 C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_void_p, C.c_size_t, C.POINTER(C.c_float), C.c_void_p]),
    "pard_cod_build_noalloc": (C.c_int, [C.c_void_p, C.POINTER(C.c_int64), C.c_int32, C.c_int32, C.c_double,
                                         C.c_double, C.c_int32, C.c_uint64, C.POINTER(C.c_int64), C.c_void_p,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "pard_rope_table_bytes": (C.c_size_t, [C.POINTER(pard_rope_spec), C.c_int32]),
    "pard_rope_table": (C.c_int, [C.POINTER(pard_rope_spec), C.c_int32, C.c_void_p, C.c_void_p]),
    "pard_qk_rope": (C.c_int, [C.POINTER(pard_rope_args), *[_HEADSP] * 4, C.c_void_p]),
    "pard_qk_rope_workspace_bytes": (C.c_size_t, [C.POINTER(pard_rope_args)]),
    "pard_qk_rope_grad": (C.c_int, [C.POINTER(pard_rope_args), *[_HEADSP] * 6, C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_size_t, C.c_void_p]),
    "pard_cod_plan_bytes": (C.c_size_t, [C.c_int64, C.c_int32]),
    "pard_cod_plan_build": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_int64), C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(pard_cod_plan)]),
    "pard_cod_attn": (C.c_int, [C.POINTER(pard_cod_attn_args), *[_HEADSP] * 4, C.c_void_p, C.c_void_p]),
    "pard_cod_attn_workspace_bytes": (C.c_size_t, [C.POINTER(pard_cod_attn_args)]),
    "pard_cod_attn_grad": (C.c_int, [C.POINTER(pard_cod_attn_args), *[_HEADSP] * 5, C.c_void_p, *[_HEADSP] * 3,
                                     C.c_void_p, C.c_size_t, C.c_void_p]),
    "pard_cod_loss_workspace_bytes": (C.c_size_t, [C.POINTER(pard_cod_loss_args)]),
    "pard_cod_loss": (C.c_int, [C.POINTER(pard_cod_loss_args), C.c_void_p, C.c_size_t, C.c_void_p]),
    "pard_read_logits": (C.c_int, [_CTX, C.c_int32, C.c_int32, C.POINTER(C.c_float), C.c_int32,
                                   C.c_int32]),
    "pard_read_weight": (C.c_int, [_CTX, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                   C.POINTER(C.c_float)]),
    "pard_timer_enable": (C.c_int, [_CTX, C.c_int32, C.c_int32]),
    "pard_timer_read": (C.c_int, [_CTX, _I32P, C.POINTER(C.c_double)]),
    "pard_last_error": (C.c_char_p, [_CTX]),
    "pard_status_string": (C.c_char_p, [C.c_int]),
    "pard_free": (None, [_CTX]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_sig)


class PardError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        name = lib.pard_status_string(status).decode()
        super().__init__(f"{name}: {message}")


def spec_from(s) -> pard_model_spec:
    """C spec from a ``pard_inputs.ModelSpec`` (the library always stores bf16)."""
    return pard_model_spec(
        n_layers=s.n_layers, d_model=s.d_model, n_heads=s.n_heads, n_kv_heads=s.n_kv_heads,
        head_dim=s.head_dim, ffn_dim=s.ffn_dim, vocab=s.vocab, rms_eps=s.rms_eps,
        rope_theta=s.rope_theta, init_std=s.init_std, qkv_bias=int(s.qkv_bias),
        tied_embeddings=int(s.tied), dtype=PARD_BF16, weight_stream=s.stream, seed=s.seed,
        **_rope_fields(s))


def _rope_fields(s) -> dict:
    if s.rope_scaling is None:
        return {}
    factor, low, high, orig = s.rope_scaling
    return dict(rope_factor=float(factor), rope_low_freq_factor=float(low), rope_high_freq_factor=float(high),
                rope_original_max_pos=int(orig))


def _i32(a) -> Tuple[np.ndarray, object]:
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return arr, arr.ctypes.data_as(_I32P)


# ---- the C calls, same names --------------------------------------------------

def pard_arena_bytes(target: pard_model_spec, draft: pard_model_spec, max_batch: int,
                     max_ctx: int, max_k: int) -> int:
    return int(lib.pard_arena_bytes(C.byref(target), C.byref(draft), max_batch, max_ctx, max_k))


def pard_model_load(target, draft, mask_id, max_batch, max_ctx, max_k, dev_arena_ptr: int,
                    arena_bytes: int, hip_stream: Optional[int]) -> int:
    ctx = _CTX()
    st = lib.pard_model_load(C.byref(target), C.byref(draft), mask_id, max_batch, max_ctx, max_k,
                             C.c_void_p(dev_arena_ptr), arena_bytes, C.c_void_p(hip_stream or 0),
                             C.byref(ctx))
    if st != PARD_OK:
        raise PardError(st, "pard_model_load failed")
    return ctx.value


def cod_capacity(n_tokens: int, k: int, r: float, r_min: float) -> int:
    return int(lib.pard_cod_capacity(int(n_tokens), int(k), float(r), float(r_min)))


def cod_build(tokens, tok_offsets: Sequence[int], k: int, r: float, r_min: float, mask_id: int, seed: int,
              stream=None, timing: bool = False):
    """COD training-data processing on the device (pard_cod_build).

    tokens: 1-D int32 device tensor of the samples back to back; tok_offsets:
    host offsets (n_samples + 1).  Returns (out_offsets, dict of the five int32
    device tensors ids/labels/pos/section/column, out_len device tensor), and
    the kernel's device milliseconds when timing is set."""
    import torch
    offs = np.ascontiguousarray(np.asarray(tok_offsets, np.int64))
    n = len(offs) - 1
    out_offs = np.zeros(max(n, 0) + 1, np.int64)
    total = lib.pard_cod_layout(offs.ctypes.data_as(C.POINTER(C.c_int64)), n, k, float(r), float(r_min),
                                out_offs.ctypes.data_as(C.POINTER(C.c_int64))) if n >= 1 else -1
    if total < 0:
        raise PardError(PARD_ERR_ARG, "cod_build: empty batch, bad parameters or a sample outside the lengths")
    dev = tokens.device
    out = {name: torch.empty(total, dtype=torch.int32, device=dev)
           for name in ("ids", "labels", "pos", "section", "column")}
    out_len = torch.empty(n, dtype=torch.int32, device=dev)
    ws_bytes = int(lib.pard_cod_workspace_bytes(n))
    ws = torch.empty(ws_bytes + 256, dtype=torch.uint8, device=dev)
    ws_ptr = ws.data_ptr() + (-ws.data_ptr()) % 256
    ms = C.c_float(0.0)
    st = stream if stream is not None else torch.cuda.current_stream(dev).cuda_stream
    rc = lib.pard_cod_build(C.c_void_p(tokens.data_ptr()), offs.ctypes.data_as(C.POINTER(C.c_int64)), n, k,
                            float(r), float(r_min), mask_id, int(seed) & ((1 << 64) - 1),
                            out_offs.ctypes.data_as(C.POINTER(C.c_int64)),
                            *[C.c_void_p(out[name].data_ptr()) for name in ("ids", "labels", "pos", "section",
                                                                            "column")],
                            C.c_void_p(out_len.data_ptr()), C.c_void_p(ws_ptr), ws_bytes,
                            C.byref(ms) if timing else None, C.c_void_p(st))
    if rc != PARD_OK:
        raise PardError(rc, "pard_cod_build failed")
    return (out_offs, out, out_len, ms.value) if timing else (out_offs, out, out_len)


PARD_COD_NOALLOC_MAX_SAMPLES = 65535


def cod_build_noalloc(tokens, tok_offsets: Sequence[int], k: int, r: float, r_min: float, mask_id: int, seed: int,
                      stream=None):
    """pard_cod_build_noalloc: as cod_build, with the offsets staged in the
    library's fixed device scratch instead of a workspace.  The output tensors
    are allocated here (by the caller of the C function)."""
    import torch
    offs = np.ascontiguousarray(np.asarray(tok_offsets, np.int64))
    n = len(offs) - 1
    out_offs = np.zeros(max(n, 0) + 1, np.int64)
    total = lib.pard_cod_layout(offs.ctypes.data_as(C.POINTER(C.c_int64)), n, k, float(r), float(r_min),
                                out_offs.ctypes.data_as(C.POINTER(C.c_int64))) if n >= 1 else -1
    if total < 0:
        raise PardError(PARD_ERR_ARG, "cod_build_noalloc: empty batch, bad parameters or a sample outside the lengths")
    dev = tokens.device
    out = {name: torch.empty(total, dtype=torch.int32, device=dev)
           for name in ("ids", "labels", "pos", "section", "column")}
    out_len = torch.empty(n, dtype=torch.int32, device=dev)
    st = stream if stream is not None else torch.cuda.current_stream(dev).cuda_stream
    rc = lib.pard_cod_build_noalloc(C.c_void_p(tokens.data_ptr()), offs.ctypes.data_as(C.POINTER(C.c_int64)), n, k,
                                    float(r), float(r_min), mask_id, int(seed) & ((1 << 64) - 1),
                                    out_offs.ctypes.data_as(C.POINTER(C.c_int64)),
                                    *[C.c_void_p(out[name].data_ptr()) for name in ("ids", "labels", "pos", "section",
                                                                                    "column")],
                                    C.c_void_p(out_len.data_ptr()), C.c_void_p(st))
    if rc != PARD_OK:
        raise PardError(rc, "pard_cod_build_noalloc failed")
    return out_offs, out, out_len


# ---- mask-token training: rotary positions, packed attention, the loss -----------

def _bad(what: str):
    raise PardError(PARD_ERR_ARG, what)


_DTYPES = {}


def _dtype(t, what: str) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: PARD_F32, torch.bfloat16: PARD_BF16, torch.float16: PARD_F16})
    if t.dtype not in _DTYPES:
        raise PardError(PARD_ERR_UNSUPPORTED, f"{what}: dtype {t.dtype}")
    return _DTYPES[t.dtype]


def _heads(t, what: str, like=None, shape=None) -> pard_heads:
    """A [rows, heads, head_dim] device tensor whose heads are contiguous."""
    st = t.stride()
    if len(st) != 3 or not t.is_cuda:
        _bad(f"{what}: a [rows, heads, head_dim] device tensor is wanted, got {tuple(t.shape)} on {t.device}")
    if st[2] != 1 and t.shape[2] > 1:
        _bad(f"{what}: the elements of a head must be contiguous")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        _bad(f"{what}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    if shape is not None and t.shape != shape:
        _bad(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    return pard_heads(t.data_ptr(), st[0], st[1])


def _vector(t, what: str, n: int, dtype, device) -> int:
    if t.dtype != dtype or t.device != device or tuple(t.shape) != (n,) or not t.is_contiguous():
        _bad(f"{what}: a contiguous {dtype} tensor of {n} on {device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _no_graph(what: str, grad_of: str) -> None:
    """Turns away tensors that require gradients where torch would record them:
    what the library returns has no graph, and a model would train without this part."""
    import torch
    if torch.is_grad_enabled():
        _bad(f"{what} records no gradient for tensors that require one: call it in a torch.autograd.Function whose "
             f"backward calls {grad_of}, or under torch.no_grad()")


class _On:
    """Runs a call on `stream` (a torch stream; None: the device's current one)
    with that device current: outputs and workspaces made inside belong to the
    stream, and `used` tensors stay alive until it is done with them."""

    __slots__ = ("handle", "stream", "ctx", "used")

    def __init__(self, device, stream, *used):
        import torch
        self.ctx = self.stream = None
        if stream is None:
            # (what torch.cuda.current_stream(device).cuda_stream is, without its Python objects)
            self.handle = torch._C._cuda_getCurrentRawStream(device.index)
            if torch._C._cuda_getDevice() != device.index:
                self.ctx = torch.cuda.device(device)
            return
        if stream.device_index != device.index:
            _bad("the stream belongs to another device than the tensors")
        self.handle, self.ctx, self.stream, self.used = stream.cuda_stream, torch.cuda.stream(stream), stream, used

    def __enter__(self):
        if self.ctx is not None:
            self.ctx.__enter__()
        return self

    def __exit__(self, *exc):
        if self.stream is not None:
            for t in self.used:
                if t is not None:
                    t.record_stream(self.stream)
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _workspace(n_bytes: int, device):
    import torch
    return torch.empty(max(n_bytes, 1), dtype=torch.uint8, device=device)   # (the allocator aligns to 512 bytes)


def _done(rc: int, what: str) -> None:
    if rc != PARD_OK:
        raise PardError(rc, f"{what} failed")


_ROPE_SCALINGS = {None: PARD_ROPE_PLAIN, "linear": PARD_ROPE_LINEAR, "llama3": PARD_ROPE_LLAMA3, "yarn": PARD_ROPE_YARN}
_ROPE_LAYOUTS = {"half": PARD_ROPE_HALF, "interleaved": PARD_ROPE_INTERLEAVED}


def rope_table(n_pos: int, rot_dim: int, theta: float, scaling: Optional[str] = None, factor: float = 1.0,
               low: float = 1.0, high: float = 4.0, original_max_pos: int = 8192, device="cuda", stream=None):
    """(cos, sin) table [n_pos, rot_dim / 2, 2] of qk_rope (pard_rope_table);
    scaling None, "linear", "llama3" or "yarn"."""
    import torch
    if scaling not in _ROPE_SCALINGS:
        _bad(f"rope_table: unknown scaling {scaling!r}")
    spec = pard_rope_spec(rot_dim, _ROPE_SCALINGS[scaling], theta, factor, low, high, original_max_pos)
    if lib.pard_rope_table_bytes(C.byref(spec), n_pos) == 0:
        _bad("rope_table: bad sizes or scaling parameters")
    device = torch.device(device)
    if device.type != "cuda":
        _bad(f"rope_table: a GPU is wanted, got {device}")
    if device.index is None:
        device = torch.device(device.type, torch.cuda.current_device())
    with _On(device, stream) as on:
        table = torch.empty(n_pos, rot_dim // 2, 2, dtype=torch.float32, device=device)
        _done(lib.pard_rope_table(C.byref(spec), n_pos, C.c_void_p(table.data_ptr()), on.handle), "pard_rope_table")
    return table


def _rope_args(q, k, positions, table, layout, q_gain, k_gain, eps) -> pard_rope_args:
    import torch
    if layout not in _ROPE_LAYOUTS:
        _bad(f"qk_rope: unknown layout {layout!r}")
    rows, n_q, hd = q.shape
    if (table.dim() != 3 or table.shape[2] != 2 or table.dtype != torch.float32 or table.device != q.device
            or not table.is_contiguous()):
        _bad("qk_rope: table: a contiguous float32 [n_pos, rot_dim / 2, 2] tensor on the queries' device is wanted")
    gains = [None if g is None else _vector(g, "gain", hd, torch.float32, q.device) for g in (q_gain, k_gain)]
    if k is not None and (q_gain is None) != (k_gain is None):
        _bad("qk_rope: both gains or neither")
    return pard_rope_args(rows, n_q, 0 if k is None else k.shape[1], hd, _dtype(q, "qk_rope"), 2 * table.shape[1],
                          _ROPE_LAYOUTS[layout], table.shape[0], eps,
                          _vector(positions, "positions", rows, torch.int32, q.device), table.data_ptr(), *gains)


def qk_rope(q, k, positions, table, layout: str = "half", q_gain=None, k_gain=None, eps: float = 1e-6, q_out=None,
            k_out=None, stream=None):
    """Rotary positions of queries and keys [rows, heads, head_dim], with gains
    after an RMSNorm of every head (pard_qk_rope).  k may be None.  Returns
    (q_out, k_out), new tensors unless given; they may be q and k themselves.
    Records no graph: where torch records gradients, tensors that require them
    are turned away (qk_rope_grad is the gradient)."""
    import torch
    if (q.requires_grad or k is not None and k.requires_grad or q_gain is not None and q_gain.requires_grad
            or k_gain is not None and k_gain.requires_grad):
        _no_graph("qk_rope", "qk_rope_grad")
    hq = _heads(q, "q")
    hk = None if k is None else _heads(k, "k", q, (*q.shape[:1], *k.shape[1:2], *q.shape[2:]))
    args = _rope_args(q, k, positions, table, layout, q_gain, k_gain, eps)
    with _On(q.device, stream, q, k, positions, table, q_gain, k_gain, q_out, k_out) as on:
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if k_out is None and k is not None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        oq = _heads(q_out, "q_out", q, q.shape)
        ok = None if k is None else _heads(k_out, "k_out", k, k.shape)
        _done(lib.pard_qk_rope(args, hq, hk, oq, ok, on.handle), "pard_qk_rope")
    return q_out, None if k is None else k_out


def qk_rope_grad(q_dy, k_dy, positions, table, layout: str = "half", q=None, k=None, q_gain=None, k_gain=None,
                 eps: float = 1e-6, q_dx=None, k_dx=None, stream=None):
    """Gradient of qk_rope (pard_qk_rope_grad).  With gains, q and k are the
    forward call's inputs.  Returns (q_dx, k_dx, q_dgain, k_dgain), the last two
    None without gains; q_dx and k_dx may be q_dy and k_dy themselves.  Every row
    counts in the gains' gradients: those of no sample need a dy of 0, finite
    heads and a position in the table."""
    import torch
    hdq = _heads(q_dy, "q_dy")
    hdk = None if k_dy is None else _heads(k_dy, "k_dy", q_dy, (*q_dy.shape[:1], *k_dy.shape[1:2], *q_dy.shape[2:]))
    args = _rope_args(q_dy, k_dy, positions, table, layout, q_gain, k_gain, eps)
    hq = hk = None
    if q_gain is not None:
        if q is None or (k_dy is not None and k is None):
            _bad("qk_rope_grad: the gradient of the norm needs the forward call's inputs")
        hq = _heads(q, "q", q_dy, q_dy.shape)
        hk = None if k_dy is None else _heads(k, "k", k_dy, k_dy.shape)
    with _On(q_dy.device, stream, q_dy, k_dy, positions, table, q, k, q_gain, k_gain, q_dx, k_dx) as on:
        new = lambda t: torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
        q_dx = new(q_dy) if q_dx is None else q_dx
        k_dx = new(k_dy) if k_dx is None and k_dy is not None else k_dx
        oq = _heads(q_dx, "q_dx", q_dy, q_dy.shape)
        ok = None if k_dy is None else _heads(k_dx, "k_dx", k_dy, k_dy.shape)
        q_dg = None if q_gain is None else new(q_gain)
        k_dg = None if q_gain is None or k_dy is None else new(k_gain) if k_dy.shape[1] else torch.zeros_like(k_gain)
        n_ws = lib.pard_qk_rope_workspace_bytes(args) if q_gain is not None else 0
        ws = _workspace(n_ws, q_dy.device) if n_ws else None
        _done(lib.pard_qk_rope_grad(args, hdq, hdk, hq, hk, oq, ok, q_dg.data_ptr() if q_dg is not None else None,
                                    k_dg.data_ptr() if k_dg is not None else None,
                                    ws.data_ptr() if n_ws else None, n_ws, on.handle), "pard_qk_rope_grad")
    return q_dx, None if k_dy is None else k_dx, q_dg, k_dg


class CodPlan:
    """Plan of a batch of packed samples (pard_cod_plan): built once per batch,
    used by every layer's cod_attn and cod_attn_grad."""

    def __init__(self, plan: pard_cod_plan, data):
        self.plan, self.data = plan, data
        self.rows, self.device = plan.rows, data.device


def cod_plan(section, column, out_offsets: Sequence[int], out_len, stream=None) -> CodPlan:
    """Plan for attention over packed rows (pard_cod_plan_build).  section,
    column, out_len: int32 device tensors as cod_build returns them,
    out_offsets: the samples' regions (host, n_samples + 1)."""
    import torch
    offs = np.ascontiguousarray(np.asarray(out_offsets, np.int64))
    n = len(offs) - 1
    if offs.ndim != 1 or n < 1 or (np.diff(offs) < 0).any() or offs[0] < 0:
        _bad("cod_plan: out_offsets must be ascending bounds of at least one sample")
    rows = int(offs[-1])
    dev = out_len.device
    for name, t in (("section", section), ("column", column)):
        if t.dtype != torch.int32 or t.device != dev or t.dim() != 1 or len(t) < rows or not t.is_contiguous():
            _bad(f"cod_plan: {name}: a contiguous int32 tensor of at least {rows} on {dev} is wanted")
    _vector(out_len, "out_len", n, torch.int32, dev)
    if dev.type != "cuda":
        _bad(f"cod_plan: device tensors are wanted, got tensors on {dev}")
    n_bytes = lib.pard_cod_plan_bytes(rows, n)
    if n_bytes == 0:
        raise PardError(PARD_ERR_UNSUPPORTED, "cod_plan: too many rows")
    plan = pard_cod_plan()
    with _On(dev, stream, section, column, out_len) as on:
        data = _workspace(n_bytes, dev)
        _done(lib.pard_cod_plan_build(section.data_ptr(), column.data_ptr(), offs.ctypes.data_as(C.POINTER(C.c_int64)),
                                      out_len.data_ptr(), n, data.data_ptr(), n_bytes, on.handle, plan),
              "pard_cod_plan_build")
    return CodPlan(plan, data)


def _attn_args(q, k, v, plan: CodPlan, scale):
    if q.dim() != 3:
        _bad(f"q: a [rows, heads, head_dim] device tensor is wanted, got {tuple(q.shape)}")
    rows, n_q, hd = q.shape
    if plan.device != q.device:
        _bad(f"cod_attn: the plan is on {plan.device}, the tensors on {q.device}")
    if rows < plan.rows:
        _bad(f"cod_attn: {rows} rows, the plan has {plan.rows}")
    shape = (rows, k.shape[1] if k.dim() == 3 else 0, hd)
    hs = _heads(q, "q"), _heads(k, "k", q, shape), _heads(v, "v", q, shape)
    scale = hd ** -0.5 if scale is None else float(scale)
    return pard_cod_attn_args(C.pointer(plan.plan), n_q, shape[1], hd, _dtype(q, "cod_attn"), scale), hs


def cod_attn(q, k, v, plan: CodPlan, scale: Optional[float] = None, out=None, stream=None):
    """Attention over packed rows (pard_cod_attn): q [rows, heads, head_dim], k
    and v [rows, kv heads, head_dim]; scale: head_dim ** -0.5 unless given.
    Returns (out, lse), lse [heads, plan rows] in float32.  Rows that belong to
    no sample's region are left as they are (out given) or hold nothing (new).
    Records no graph, as qk_rope (cod_attn_grad is the gradient)."""
    import torch
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _no_graph("cod_attn", "cod_attn_grad")
    args, (hq, hk, hv) = _attn_args(q, k, v, plan, scale)
    with _On(q.device, stream, q, k, v, plan.data, out) as on:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        ho = _heads(out, "out", q, q.shape)
        lse = torch.empty(q.shape[1], plan.rows, dtype=torch.float32, device=q.device)
        _done(lib.pard_cod_attn(args, hq, hk, hv, ho, lse.data_ptr(), on.handle), "pard_cod_attn")
    return out, lse


def cod_attn_grad(d_out, q, k, v, out, lse, plan: CodPlan, scale: Optional[float] = None, dq=None, dk=None, dv=None,
                  stream=None):
    """Gradient of cod_attn (pard_cod_attn_grad); out and lse are the forward
    call's.  Returns (dq, dk, dv), new tensors unless given."""
    import torch
    args, (hq, hk, hv) = _attn_args(q, k, v, plan, scale)
    hdo, ho = _heads(d_out, "d_out", q, q.shape), _heads(out, "out", q, q.shape)
    if (lse.dtype != torch.float32 or lse.device != q.device or tuple(lse.shape) != (q.shape[1], plan.rows)
            or not lse.is_contiguous()):
        _bad(f"cod_attn_grad: lse: the forward call's ({q.shape[1]}, {plan.rows}) tensor is wanted")
    with _On(q.device, stream, d_out, q, k, v, out, lse, plan.data, dq, dk, dv) as on:
        new = lambda t: torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
        dq, dk, dv = (new(t) if d is None else d for d, t in ((dq, q), (dk, k), (dv, v)))
        outs = [_heads(d, n, t, t.shape) for d, n, t in ((dq, "dq", q), (dk, "dk", k), (dv, "dv", v))]
        n_ws = lib.pard_cod_attn_workspace_bytes(args)
        ws = _workspace(n_ws, q.device)
        _done(lib.pard_cod_attn_grad(args, hdo, hq, hk, hv, ho, lse.data_ptr(), *outs, ws.data_ptr(), n_ws, on.handle),
              "pard_cod_attn_grad")
    return dq, dk, dv


def cod_loss(logits, labels, section, n_sections: int, weights: Optional[Sequence[float]] = None, grad: bool = True,
             grad_scale: float = 1.0, d_logits=None, stream=None):
    """Mask-token loss of logits [rows, vocab] and its gradient (pard_cod_loss).
    labels, section: int32 [rows] (cod_build's; section None: one subtask);
    weights: of the subtasks' means, None: the mean over all counted rows.
    Returns (loss [], subtask means [n_sections], row losses [rows], d_logits or
    None); d_logits may be logits itself.  The loss has no graph: gradients go on
    from d_logits (logits.backward(d_logits))."""
    import torch
    if logits.dim() != 2 or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        _bad("cod_loss: logits: a [rows, vocab] device tensor with contiguous rows is wanted")
    rows, vocab = logits.shape
    dev = logits.device
    w = None
    if weights is not None:
        if len(weights) != n_sections:
            _bad(f"cod_loss: {len(weights)} weights for {n_sections} subtasks")
        w = (C.c_float * max(n_sections, 1))(*[float(x) for x in weights])
    p_labels = _vector(labels, "labels", rows, torch.int32, dev)
    p_section = None if section is None else _vector(section, "section", rows, torch.int32, dev)
    if not 1 <= n_sections <= 64:
        _bad("cod_loss: n_sections outside [1, 64]")
    with _On(dev, stream, logits, labels, section, d_logits) as on:
        if grad and d_logits is None:
            d_logits = torch.empty(rows, vocab, dtype=logits.dtype, device=dev)
        if not grad:
            d_logits = None
        elif (d_logits.dtype != logits.dtype or d_logits.device != dev or d_logits.shape != logits.shape
              or (vocab > 1 and d_logits.stride(1) != 1)):
            _bad("cod_loss: d_logits: a tensor like logits is wanted")
        loss = torch.empty(1 + n_sections, dtype=torch.float32, device=dev)
        row_loss = torch.empty(rows, dtype=torch.float32, device=dev)
        args = pard_cod_loss_args(rows, vocab, _dtype(logits, "cod_loss"), n_sections, grad_scale, logits.data_ptr(),
                                  logits.stride(0), p_labels, p_section, w, None if d_logits is None else d_logits.data_ptr(),
                                  0 if d_logits is None else d_logits.stride(0), loss.data_ptr(), row_loss.data_ptr())
        n_ws = lib.pard_cod_loss_workspace_bytes(args)
        ws = _workspace(n_ws, dev)
        _done(lib.pard_cod_loss(args, ws.data_ptr(), n_ws, on.handle), "pard_cod_loss")
    return loss[0], loss[1:], row_loss, d_logits


class Engine:
    """A loaded target/draft pair: owns the torch arena and the context."""

    def __init__(self, target_spec, draft_spec, mask_id: int, max_ctx: int, max_k: int,
                 max_batch: int = 1, device: str = "cuda:0", stream=None):
        import torch
        self.target_spec, self.draft_spec = target_spec, draft_spec
        self.vocab = target_spec.vocab
        self.mask_id = mask_id
        self._t, self._d = spec_from(target_spec), spec_from(draft_spec)
        nbytes = pard_arena_bytes(self._t, self._d, max_batch, max_ctx, max_k)
        if nbytes == 0:
            raise PardError(PARD_ERR_ARG, "invalid specs or capacities")
        self.device = torch.device(device)
        self.arena = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.arena.data_ptr()
        base += (-base) % 256
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self.ctx = pard_model_load(self._t, self._d, mask_id, max_batch, max_ctx, max_k, base,
                                   nbytes, self.stream.cuda_stream)
        self.max_ctx, self.max_k, self.max_batch = max_ctx, max_k, max_batch

    def close(self) -> None:
        if getattr(self, "ctx", None):
            lib.pard_free(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, what: str) -> None:
        if st != PARD_OK:
            raise PardError(st, f"{what}: {lib.pard_last_error(self.ctx).decode()}")

    def prefill(self, prompt: Sequence[int], seq: int = 0) -> int:
        arr, ptr = _i32(prompt)
        first = C.c_int32()
        self._check(lib.pard_prefill(self.ctx, seq, ptr, len(arr), C.byref(first)), "pard_prefill")
        return first.value

    def draft(self, prefix: Sequence[int], k: int, seq: int = 0) -> list:
        arr, ptr = _i32(prefix)
        out = np.zeros(max(k, 1), np.int32)
        self._check(lib.pard_draft(self.ctx, seq, ptr, len(arr), k, out.ctypes.data_as(_I32P)),
                    "pard_draft")
        return [int(x) for x in out[:k]]

    def verify(self, cand: Sequence[int], seq: int = 0) -> Tuple[int, int]:
        arr, ptr = _i32(list(cand) if len(cand) else [0])
        a, bonus = C.c_int32(), C.c_int32()
        self._check(lib.pard_verify(self.ctx, seq, ptr, len(cand), C.byref(a), C.byref(bonus)),
                    "pard_verify")
        return a.value, bonus.value

    def set_sampling(self, temperature: float, seed: int = 0) -> None:
        """Speculative sampling at temperature T > 0 for later calls; 0 = greedy."""
        self._check(lib.pard_set_sampling(self.ctx, float(temperature), int(seed) & ((1 << 64) - 1)),
                    "pard_set_sampling")

    def kv_len(self, which: int, seq: int = 0) -> int:
        n = C.c_int32()
        self._check(lib.pard_kv_len(self.ctx, seq, which, C.byref(n)), "pard_kv_len")
        return n.value

    def kv_truncate(self, which: int, new_len: int, seq: int = 0) -> None:
        self._check(lib.pard_kv_truncate(self.ctx, seq, which, new_len), "pard_kv_truncate")

    def generate(self, k: int, n_tokens: int, max_steps: int = 0, seq: int = 0,
                 mode: int = PARD_MODE_PARALLEL):
        out = np.zeros(n_tokens, np.int32)
        stats = pard_stats()
        seqs, sptr = _i32([seq])
        self._check(lib.pard_generate_ex(self.ctx, 1, sptr, k, mode, n_tokens, max_steps,
                                         out.ctypes.data_as(_I32P), C.byref(stats)), "pard_generate_ex")
        return out[:stats.tokens].tolist(), stats

    def generate_batch(self, seqs: Sequence[int], k: int, n_tokens: int, max_steps: int = 0,
                       mode: int = PARD_MODE_PARALLEL):
        """Fused loop over several slots at once (batched passes).  Returns one
        token list per slot (the pending token first) and the summed stats."""
        before = [self.kv_len(PARD_TARGET, seq=s) for s in seqs]
        out = np.zeros((len(seqs), n_tokens), np.int32)
        stats = pard_stats()
        arr, sptr = _i32(list(seqs))
        self._check(lib.pard_generate_ex(self.ctx, len(seqs), sptr, k, mode, n_tokens, max_steps,
                                         out.ctypes.data_as(_I32P), C.byref(stats)), "pard_generate_ex")
        res = []
        for i, s in enumerate(seqs):
            n = min(n_tokens, 1 + self.kv_len(PARD_TARGET, seq=s) - before[i])
            res.append(out[i, :n].tolist())
        return res, stats

    def read_logits(self, which: int, rows: int, seq: int = 0) -> np.ndarray:
        out = np.zeros((rows, self.vocab), np.float32)
        self._check(lib.pard_read_logits(self.ctx, which, seq,
                                         out.ctypes.data_as(C.POINTER(C.c_float)), rows,
                                         self.vocab), "pard_read_logits")
        return out

    def read_weight(self, which: int, tensor: int, row: int, col0: int, n: int) -> np.ndarray:
        out = np.zeros(n, np.float32)
        self._check(lib.pard_read_weight(self.ctx, which, tensor, row, col0, n,
                                         out.ctypes.data_as(C.POINTER(C.c_float))),
                    "pard_read_weight")
        return out

    def timer_enable(self, kernel_class: int, max_launches: int) -> None:
        self._check(lib.pard_timer_enable(self.ctx, kernel_class, max_launches), "pard_timer_enable")

    def timer_read(self) -> Tuple[int, float]:
        n, ms = C.c_int32(), C.c_double()
        self._check(lib.pard_timer_read(self.ctx, C.byref(n), C.byref(ms)), "pard_timer_read")
        return n.value, ms.value
