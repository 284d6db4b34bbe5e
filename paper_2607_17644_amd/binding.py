"""ctypes binding of include/laga.h (marshalling only; torch supplies memory and streams).

Each ``laga_*`` function takes torch tensors, checks dtype/shape/device/
contiguity, passes raw pointers and the current HIP stream to the C entry point
of the same name, and raises :class:`LagaError` on a non-zero status. Outputs and
workspaces that are not supplied are allocated with torch (the C library never allocates),
on the stream that the call runs on; where that is not the current one (``stream=``), outputs are kept
from reuse until the current stream, too, has done what it was given before they were dropped.
"""
from __future__ import annotations

import ctypes
import dataclasses
import functools
import inspect
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_PKG, "liblaga.so")

DTYPE_BF16, DTYPE_FP32 = 0, 1
DQ_FROM_STORE, DQ_RECOMPUTE = 0, 1
KV_MATERIALIZED, KV_FUSED = 0, 1
OP_FWD, OP_BWD, OP_PROLOGUE_BWD = 0, 1, 2
OP_PAGE_PLAN, OP_PAGED_ATTN, OP_PAGED_ATTN_Q8 = 3, 4, 5  # laga_paged_workspace_bytes
PLAN_ROWS, PLAN_TABLE, PLAN_PAGES, PLAN_INVALID = 1, 2, 4, 8  # bits of a plan's status
BWD_PREPARE, BWD_DKDV, BWD_DQ, BWD_FINISH = 0, 1, 2, 3

_STATUS = {0: "LAGA_OK", 1: "LAGA_ERR_NULL", 2: "LAGA_ERR_SHAPE", 3: "LAGA_ERR_UNSUPPORTED",
           4: "LAGA_ERR_ALIGN", 5: "LAGA_ERR_WORKSPACE", 6: "LAGA_ERR_DEVICE", 7: "LAGA_ERR_SCRATCH"}
NOALLOC_SCRATCH_BYTES = 128 << 20  # LAGA_NOALLOC_SCRATCH_BYTES


class LagaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {laga_status_string(status)}")


class _CProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seq_len", ctypes.c_int64), ("n_heads", ctypes.c_int64),
                ("d_c", ctypes.c_int64), ("d_nope", ctypes.c_int64), ("d_rope", ctypes.c_int64),
                ("d_v", ctypes.c_int64), ("softmax_scale", ctypes.c_float), ("causal", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("kv_mode", ctypes.c_int32), ("deterministic", ctypes.c_int32),
                ("dq_mode", ctypes.c_int32)]


class _COutProj(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("n_heads", ctypes.c_int64), ("d_v", ctypes.c_int64),
                ("d_model", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


@dataclasses.dataclass
class OutProj:
    """Mirror of laga_out_proj_t (Alg. 1 step 7: y = reshape(out) @ w_o)."""
    tokens: int
    n_heads: int
    d_v: int
    d_model: int
    dtype: int = DTYPE_BF16
    reserved: int = 0

    def c(self) -> _COutProj:
        return _COutProj(self.tokens, self.n_heads, self.d_v, self.d_model, self.dtype, self.reserved)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == DTYPE_BF16 else torch.float32

    def shapes(self) -> dict:
        T, F = self.tokens, self.n_heads * self.d_v
        return {"out": (T, self.n_heads, self.d_v), "w_o": (F, self.d_model), "y": (T, self.d_model),
                "dy": (T, self.d_model), "d_out": (T, self.n_heads, self.d_v), "dw_o": (F, self.d_model)}


class _CPrologue(ctypes.Structure):
    _fields_ = [("eps", ctypes.c_float), ("rope_base", ctypes.c_float), ("position_offset", ctypes.c_int64)]


class _CPaged(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "requests", "table_width", "n_pages", "page_size",
                                              "page_stride", "n_heads", "d_c", "d_nope", "d_rope", "d_v")] + [
        ("softmax_scale", ctypes.c_float), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


@dataclasses.dataclass
class Paged:
    """Mirror of laga_paged_t: one serving step over a paged cache of latents."""
    rows: int         # new tokens of the step, rows of padding included
    requests: int
    table_width: int  # block-table entries of a request
    n_pages: int
    page_size: int
    n_heads: int
    d_c: int
    d_nope: int
    d_rope: int
    d_v: int
    softmax_scale: float
    dtype: int = DTYPE_BF16
    page_stride: int = 0  # elements between pages; 0: pages are contiguous
    reserved: int = 0

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        self.__dict__.pop("_made", None)  # what was made of the fields before

    def __getstate__(self):
        """The fields: a reference into C memory is neither copied nor pickled."""
        return {k: v for k, v in self.__dict__.items() if k != "_made"}

    def _forms(self):
        """(reference to the C struct, shapes), made once for these fields: a step passes them to each call."""
        made = self.__dict__.get("_made")
        if made is None:
            made = self.__dict__["_made"] = (ctypes.byref(self.c()), self._shapes())
        return made

    def ref(self):
        return self._forms()[0]

    def shapes(self) -> dict:
        return self._forms()[1]

    def c(self) -> _CPaged:
        return _CPaged(self.rows, self.requests, self.table_width, self.n_pages, self.page_size, self.page_stride,
                       self.n_heads, self.d_c, self.d_nope, self.d_rope, self.d_v, self.softmax_scale, self.dtype,
                       self.reserved)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == DTYPE_BF16 else torch.float32

    def _shapes(self) -> dict:
        T, R, H = self.rows, self.requests, self.n_heads
        return {"gamma": (self.d_c,), "cache": (self.n_pages, self.page_size, self.d_c + self.d_rope), "block_table": (R, self.table_width),
                "scales": (self.n_pages, self.page_size, 2), "c_kv": (T, self.d_c), "k_pe": (T, self.d_rope),
                "free_pages": (self.n_pages,), "free_count": (1,), "free_count_out": (1,), "status": (1,),
                "lengths": (R,), "lengths_out": (R,), "fresh": (R,), "drop": (R,), "row_begin": (R + 1,),
                "row_request": (T,), "position": (T,), "slot": (T,), "latent_raw": (T, self.d_c),
                "kpe_raw": (T, self.d_rope), "q": (T, H, self.d_nope + self.d_rope),
                "w_kv_b": (self.d_c, H * (self.d_nope + self.d_v)), "out": (T, H, self.d_v), "lse": (T, H)}


@dataclasses.dataclass
class Problem:
    """Mirror of laga_problem_t."""
    batch: int
    seq_len: int
    n_heads: int
    d_c: int
    d_nope: int
    d_rope: int
    d_v: int
    softmax_scale: float  # multiplies q.k; the caller chooses it (the library has no default)
    causal: int = 1
    dtype: int = DTYPE_BF16
    kv_mode: int = KV_MATERIALIZED
    deterministic: int = 1
    dq_mode: int = DQ_FROM_STORE

    def c(self) -> _CProblem:
        return _CProblem(self.batch, self.seq_len, self.n_heads, self.d_c, self.d_nope, self.d_rope,
                         self.d_v, self.softmax_scale, self.causal, self.dtype, self.kv_mode,
                         self.deterministic, self.dq_mode)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == DTYPE_BF16 else torch.float32

    def shapes(self) -> dict:
        B, S, H = self.batch, self.seq_len, self.n_heads
        dqk, dkvh = self.d_nope + self.d_rope, self.d_nope + self.d_v
        return {"c_kv": (B, S, self.d_c), "k_pe": (B, S, self.d_rope), "q": (B, S, H, dqk),
                "w_kv_b": (self.d_c, H * dkvh), "kv": (B, S, H, dkvh), "out": (B, S, H, self.d_v),
                "lse": (B, H, S), "dout": (B, S, H, self.d_v), "dq": (B, S, H, dqk),
                "dc_kv": (B, S, self.d_c), "dk_pe": (B, S, self.d_rope), "dw_kv_b": (self.d_c, H * dkvh)}


def _load():
    if not os.path.exists(lib_path):
        raise ImportError(f"{lib_path} is not built; run `python paper_2607_17644_amd/build.py`")
    L = ctypes.CDLL(lib_path)
    vp, P = ctypes.c_void_p, ctypes.POINTER(_CProblem)
    L.laga_abi_version.restype = ctypes.c_int
    L.laga_status_string.restype = ctypes.c_char_p
    L.laga_status_string.argtypes = [ctypes.c_int]
    L.laga_workspace_bytes.restype = ctypes.c_size_t
    L.laga_workspace_bytes.argtypes = [P, ctypes.c_int]
    L.laga_reconstruct_kv.restype = ctypes.c_int
    L.laga_reconstruct_kv.argtypes = [P, vp, vp, vp, vp]
    L.laga_attn_fwd.restype = ctypes.c_int
    L.laga_attn_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.laga_attn_bwd.restype = ctypes.c_int
    L.laga_attn_bwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.laga_attn_bwd_noalloc.restype = ctypes.c_int
    L.laga_attn_bwd_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.laga_attn_bwd_stage.restype = ctypes.c_int
    L.laga_attn_bwd_stage.argtypes = [ctypes.c_int, P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                      ctypes.c_size_t, vp]
    O = ctypes.POINTER(_COutProj)
    L.laga_out_proj_fwd.restype = ctypes.c_int
    L.laga_out_proj_fwd.argtypes = [O, vp, vp, vp, vp]
    L.laga_out_proj_bwd.restype = ctypes.c_int
    L.laga_out_proj_bwd.argtypes = [O, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    L.laga_out_proj_workspace_bytes.restype = ctypes.c_size_t
    L.laga_out_proj_workspace_bytes.argtypes = [O]
    Q = ctypes.POINTER(_CPrologue)
    L.laga_prologue_fwd.restype = ctypes.c_int
    L.laga_prologue_fwd.argtypes = [P, Q, vp, vp, vp, vp, vp, vp, vp, vp]
    L.laga_prologue_bwd.restype = ctypes.c_int
    L.laga_prologue_bwd.argtypes = [P, Q, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    G = ctypes.POINTER(_CPaged)
    L.laga_paged_workspace_bytes.restype = ctypes.c_size_t
    L.laga_paged_workspace_bytes.argtypes = [G, ctypes.c_int]
    L.laga_page_plan.restype = ctypes.c_int
    L.laga_page_plan.argtypes = [G] + [vp] * 13 + [ctypes.c_size_t, vp]
    L.laga_page_release.restype = ctypes.c_int
    L.laga_page_release.argtypes = [G] + [vp] * 9 + [ctypes.c_size_t, vp]
    L.laga_cache_append.restype = ctypes.c_int
    L.laga_cache_append.argtypes = [G, Q, vp, ctypes.c_int64, vp, vp, ctypes.c_int64, vp, vp, vp, vp]
    L.laga_paged_attn.restype = ctypes.c_int
    L.laga_paged_attn.argtypes = [G, Q] + [vp] * 9 + [ctypes.c_size_t, vp]
    L.laga_cache_append_q8.restype = ctypes.c_int
    L.laga_cache_append_q8.argtypes = [G, Q, vp, ctypes.c_int64, vp, vp, ctypes.c_int64, vp, vp, vp, vp, vp]
    L.laga_cache_read_q8.restype = ctypes.c_int
    L.laga_cache_read_q8.argtypes = [G] + [vp] * 8
    L.laga_paged_attn_q8.restype = ctypes.c_int
    L.laga_paged_attn_q8.argtypes = [G, Q] + [vp] * 10 + [ctypes.c_size_t, vp]
    return L


_lib = _load()


def laga_abi_version() -> int:
    return _lib.laga_abi_version()


def laga_status_string(status: int) -> str:
    return _lib.laga_status_string(status).decode()


def laga_workspace_bytes(p: Problem, op: int) -> int:
    return int(_lib.laga_workspace_bytes(ctypes.byref(p.c()), op))


def _ptr(t, name, shape=None, dtype=None, required=True):
    if t is None:
        if required:
            raise ValueError(f"{name} is required")
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _kept(tensors, stream):
    """Outputs allocated on `stream` and handed to the caller, whose own work is on the current stream."""
    now = torch.cuda.current_stream(stream.device)
    if now != stream:
        for t in tensors:
            t.record_stream(now)


def _on_its_stream(call):
    """What the call allocates belongs to the stream that it runs on. (A block of another stream's could be
    dropped, as a workspace is on return, and given out again there while the call still uses it.)"""
    at = list(inspect.signature(call).parameters).index("stream")

    @functools.wraps(call)
    def on_its_stream(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return call(*args, **kw)
        with torch.cuda.stream(stream):
            result = call(*args, **kw)
        _kept([t for t in (result if isinstance(result, (tuple, list)) else (result,)) if isinstance(t, torch.Tensor)], stream)
        return result

    return on_its_stream


def _check(status, where):
    if status != 0:
        raise LagaError(status, where)


def _new(p, name, dtype, device):
    return torch.empty(p.shapes()[name], dtype=dtype, device=device)


@_on_its_stream
def laga_reconstruct_kv(p: Problem, c_kv, w_kv_b, kv=None, stream=None):
    """kv = c_kv @ w_kv_b as [B,S,H,d_nope+d_v] (Alg. 1 step 4)."""
    sh, dt = p.shapes(), p.torch_dtype
    if kv is None:
        kv = _new(p, "kv", dt, c_kv.device)
    _check(_lib.laga_reconstruct_kv(ctypes.byref(p.c()), _ptr(c_kv, "c_kv", sh["c_kv"], dt),
                                    _ptr(w_kv_b, "w_kv_b", sh["w_kv_b"], dt),
                                    _ptr(kv, "kv", sh["kv"], dt), _stream(stream)), "laga_reconstruct_kv")
    return kv


def _workspace(p, op, workspace, device):
    need = laga_workspace_bytes(p, op)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    return workspace


@_on_its_stream
def laga_attn_fwd(p: Problem, q, c_kv, k_pe, w_kv_b, kv=None, out=None, lse=None, workspace=None,
                  stream=None):
    """Causal MLA attention forward of the shard's heads; returns (out, lse)."""
    sh, dt = p.shapes(), p.torch_dtype
    dev = q.device
    if out is None:
        out = _new(p, "out", dt, dev)
    if lse is None:
        lse = _new(p, "lse", torch.float32, dev)
    workspace = _workspace(p, OP_FWD, workspace, dev)
    _check(_lib.laga_attn_fwd(
        ctypes.byref(p.c()), _ptr(q, "q", sh["q"], dt), _ptr(c_kv, "c_kv", sh["c_kv"], dt),
        _ptr(k_pe, "k_pe", sh["k_pe"], dt), _ptr(w_kv_b, "w_kv_b", sh["w_kv_b"], dt),
        _ptr(kv, "kv", sh["kv"], dt, required=False), _ptr(out, "out", sh["out"], dt),
        _ptr(lse, "lse", sh["lse"], torch.float32), _ptr(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(stream)), "laga_attn_fwd")
    return out, lse


def _bwd_args(p, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq, dc_kv, dk_pe, dw_kv_b, workspace):
    sh, dt = p.shapes(), p.torch_dtype
    return (ctypes.byref(p.c()), _ptr(q, "q", sh["q"], dt), _ptr(c_kv, "c_kv", sh["c_kv"], dt),
            _ptr(k_pe, "k_pe", sh["k_pe"], dt), _ptr(w_kv_b, "w_kv_b", sh["w_kv_b"], dt),
            _ptr(kv, "kv", sh["kv"], dt, required=False), _ptr(out, "out", sh["out"], dt),
            _ptr(lse, "lse", sh["lse"], torch.float32), _ptr(dout, "dout", sh["dout"], dt),
            _ptr(dq, "dq", sh["dq"], dt), _ptr(dc_kv, "dc_kv", sh["dc_kv"], torch.float32),
            _ptr(dk_pe, "dk_pe", sh["dk_pe"], torch.float32),
            _ptr(dw_kv_b, "dw_kv_b", sh["dw_kv_b"], torch.float32),
            _ptr(workspace, "workspace", required=False),
            0 if workspace is None else workspace.numel() * workspace.element_size())


def _bwd_outputs(p, dev, dq, dc_kv, dk_pe, dw_kv_b, workspace):
    if dq is None:
        dq = _new(p, "dq", p.torch_dtype, dev)
    if dc_kv is None:
        dc_kv = _new(p, "dc_kv", torch.float32, dev)
    if dk_pe is None:
        dk_pe = _new(p, "dk_pe", torch.float32, dev)
    if dw_kv_b is None:
        dw_kv_b = _new(p, "dw_kv_b", torch.float32, dev)
    workspace = _workspace(p, OP_BWD, workspace, dev)
    return dq, dc_kv, dk_pe, dw_kv_b, workspace


@_on_its_stream
def laga_attn_bwd(p: Problem, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq=None, dc_kv=None,
                  dk_pe=None, dw_kv_b=None, workspace=None, stream=None):
    """Backward of the block; returns (dq, dc_kv, dk_pe, dw_kv_b) — dq in the element
    dtype, the head-shard partials dc_kv / dk_pe and dw_kv_b in fp32."""
    dq, dc_kv, dk_pe, dw_kv_b, workspace = _bwd_outputs(p, q.device, dq, dc_kv, dk_pe, dw_kv_b, workspace)
    _check(_lib.laga_attn_bwd(*_bwd_args(p, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq, dc_kv, dk_pe,
                                         dw_kv_b, workspace), _stream(stream)), "laga_attn_bwd")
    return dq, dc_kv, dk_pe, dw_kv_b


@_on_its_stream
def laga_attn_bwd_noalloc(p: Problem, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq=None, dc_kv=None,
                          dk_pe=None, dw_kv_b=None, stream=None):
    """laga_attn_bwd with the library's fixed device scratch array as its workspace (for
    callers that cannot allocate; LagaError LAGA_ERR_SCRATCH above its size). Outputs not
    supplied are allocated here, as for laga_attn_bwd."""
    dev = q.device
    dq, dc_kv, dk_pe, dw_kv_b = [t if t is not None else _new(p, n, dt, dev) for t, n, dt in (
        (dq, "dq", p.torch_dtype), (dc_kv, "dc_kv", torch.float32), (dk_pe, "dk_pe", torch.float32),
        (dw_kv_b, "dw_kv_b", torch.float32))]
    args = _bwd_args(p, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq, dc_kv, dk_pe, dw_kv_b, None)
    _check(_lib.laga_attn_bwd_noalloc(*args[:-2], _stream(stream)), "laga_attn_bwd_noalloc")
    return dq, dc_kv, dk_pe, dw_kv_b


def laga_attn_bwd_stage(stage: int, p: Problem, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq, dc_kv,
                        dk_pe, dw_kv_b, workspace, stream=None):
    """One stage of laga_attn_bwd (BWD_PREPARE, BWD_DKDV, BWD_DQ, BWD_FINISH); all buffers
    must be supplied and be the same for every stage of one backward."""
    _check(_lib.laga_attn_bwd_stage(stage, *_bwd_args(p, q, c_kv, k_pe, w_kv_b, kv, out, lse, dout, dq,
                                                       dc_kv, dk_pe, dw_kv_b, workspace), _stream(stream)),
           "laga_attn_bwd_stage")


def laga_out_proj_workspace_bytes(p: OutProj) -> int:
    return int(_lib.laga_out_proj_workspace_bytes(ctypes.byref(p.c())))


@_on_its_stream
def laga_out_proj_fwd(p: OutProj, out, w_o, y=None, stream=None):
    """Alg. 1 step 7: y = reshape(out) @ w_o; out [T, n_heads, d_v], w_o [F, d_model]."""
    sh, dt = p.shapes(), p.torch_dtype
    if y is None:
        y = torch.empty(sh["y"], dtype=dt, device=out.device)
    _check(_lib.laga_out_proj_fwd(ctypes.byref(p.c()), _ptr(out, "out", sh["out"], dt),
                                  _ptr(w_o, "w_o", sh["w_o"], dt), _ptr(y, "y", sh["y"], dt), _stream(stream)),
           "laga_out_proj_fwd")
    return y


@_on_its_stream
def laga_out_proj_bwd(p: OutProj, out, w_o, dy, d_out=None, dw_o=None, workspace=None, stream=None):
    """Backward of laga_out_proj_fwd: (d_out in the element dtype, dw_o in fp32)."""
    sh, dt = p.shapes(), p.torch_dtype
    dev = out.device
    if d_out is None:
        d_out = torch.empty(sh["d_out"], dtype=dt, device=dev)
    if dw_o is None:
        dw_o = torch.empty(sh["dw_o"], dtype=torch.float32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(1, laga_out_proj_workspace_bytes(p)), dtype=torch.uint8, device=dev)
    _check(_lib.laga_out_proj_bwd(ctypes.byref(p.c()), _ptr(out, "out", sh["out"], dt),
                                  _ptr(w_o, "w_o", sh["w_o"], dt), _ptr(dy, "dy", sh["dy"], dt),
                                  _ptr(d_out, "d_out", sh["d_out"], dt),
                                  _ptr(dw_o, "dw_o", sh["dw_o"], torch.float32), _ptr(workspace, "workspace"),
                                  workspace.numel() * workspace.element_size(), _stream(stream)),
           "laga_out_proj_bwd")
    return d_out, dw_o


@_on_its_stream
def laga_prologue_fwd(p: Problem, latent_raw, kpe_raw, q=None, gamma=None, eps=1e-6, rope_base=10000.0,
                      position_offset=0, c_kv=None, k_pe=None, rstd=None, stream=None):
    """Latent normalisation and decoupled RoPE before the all-gather; returns (c_kv, k_pe,
    rstd). The q_rope columns of q (if given) are rotated in place."""
    sh, dt = p.shapes(), p.torch_dtype
    dev = latent_raw.device
    if c_kv is None:
        c_kv = _new(p, "c_kv", dt, dev)
    if k_pe is None:
        k_pe = _new(p, "k_pe", dt, dev)
    if rstd is None:
        rstd = torch.empty((p.batch, p.seq_len), dtype=torch.float32, device=dev)
    cfg = _CPrologue(eps, rope_base, position_offset)
    _check(_lib.laga_prologue_fwd(
        ctypes.byref(p.c()), ctypes.byref(cfg), _ptr(latent_raw, "latent_raw", sh["c_kv"], dt),
        _ptr(gamma, "gamma", (p.d_c,), dt, required=False), _ptr(kpe_raw, "kpe_raw", sh["k_pe"], dt),
        _ptr(q, "q", sh["q"], dt, required=False), _ptr(c_kv, "c_kv", sh["c_kv"], dt),
        _ptr(k_pe, "k_pe", sh["k_pe"], dt), _ptr(rstd, "rstd", (p.batch, p.seq_len), torch.float32),
        _stream(stream)), "laga_prologue_fwd")
    return c_kv, k_pe, rstd


@_on_its_stream
def laga_prologue_bwd(p: Problem, latent_raw, rstd, dc_kv, dk_pe, dq=None, gamma=None, eps=1e-6,
                      rope_base=10000.0, position_offset=0, d_latent_raw=None, d_kpe_raw=None, d_gamma=None,
                      workspace=None, stream=None):
    """Backward of laga_prologue_fwd; returns (d_latent_raw, d_kpe_raw, d_gamma) in fp32
    (d_gamma None without gamma). The q_rope columns of dq (if given) are rotated back in place."""
    sh, dt = p.shapes(), p.torch_dtype
    dev = latent_raw.device
    if d_latent_raw is None:
        d_latent_raw = _new(p, "dc_kv", torch.float32, dev)
    if d_kpe_raw is None:
        d_kpe_raw = _new(p, "dk_pe", torch.float32, dev)
    if gamma is not None and d_gamma is None:
        d_gamma = torch.empty((p.d_c,), dtype=torch.float32, device=dev)
    nbytes = 0
    if gamma is not None:
        workspace = _workspace(p, OP_PROLOGUE_BWD, workspace, dev)
        nbytes = workspace.numel() * workspace.element_size()
    cfg = _CPrologue(eps, rope_base, position_offset)
    _check(_lib.laga_prologue_bwd(
        ctypes.byref(p.c()), ctypes.byref(cfg), _ptr(latent_raw, "latent_raw", sh["c_kv"], dt),
        _ptr(gamma, "gamma", (p.d_c,), dt, required=False),
        _ptr(rstd, "rstd", (p.batch, p.seq_len), torch.float32),
        _ptr(dc_kv, "dc_kv", sh["dc_kv"], torch.float32), _ptr(dk_pe, "dk_pe", sh["dk_pe"], torch.float32),
        _ptr(dq, "dq", sh["dq"], dt, required=False),
        _ptr(d_latent_raw, "d_latent_raw", sh["dc_kv"], torch.float32),
        _ptr(d_kpe_raw, "d_kpe_raw", sh["dk_pe"], torch.float32),
        _ptr(d_gamma, "d_gamma", (p.d_c,), torch.float32, required=gamma is not None),
        _ptr(workspace, "workspace", required=False), nbytes, _stream(stream)), "laga_prologue_bwd")
    return d_latent_raw, d_kpe_raw, d_gamma


def laga_paged_workspace_bytes(p: Paged, op: int) -> int:
    return int(_lib.laga_paged_workspace_bytes(p.ref(), op))


def _fault(t, name, shape, dtype, index):
    """Why t is not a contiguous tensor of this shape and type on device number index."""
    if not isinstance(t, torch.Tensor):
        return TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        return ValueError(f"{name} must be a device tensor")
    if t.get_device() != index:
        return ValueError(f"{name} is on {t.device}, expected cuda:{index}")
    if tuple(t.shape) != shape:
        return ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    if t.dtype != dtype:
        return ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    return ValueError(f"{name} must be contiguous")


def _at(t, name, shape, dtype, index):
    """Address of a required contiguous tensor. (A decoding step makes some thirty of these checks, and its
    kernels take microseconds: what is right is found right at once, what is not is looked at again.)"""
    try:
        if t.shape == shape and t.dtype is dtype and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    raise _fault(t, name, shape, dtype, index)


def _device_of(t, name):
    """Number of the device of a serving call: that of its first tensor; every other has to be on it."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    index = t.get_device()
    if index < 0:
        raise ValueError(f"{name} must be a device tensor")
    return index


def _rows_at(t, name, shape, dtype, index):
    """Address and row stride of a matrix whose rows are contiguous (columns of a wider one)."""
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise _fault(t, name, shape, dtype, index)
    if t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]


def _cache_at(p, t, index, dtype=None):
    """Address of the pool: rows contiguous in a page, pages p.page_stride elements apart."""
    shape, dtype = p.shapes()["cache"], dtype or p.torch_dtype
    if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        raise _fault(t, "cache", shape, dtype, index)
    want = (p.page_stride or shape[1] * shape[2], shape[2], 1)
    if t.stride() != want and any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), want)):
        raise ValueError(f"cache has strides {t.stride()}, expected {want}")
    return t.data_ptr()


def _serve(where, index, stream, function, *args):
    """The call with its device current, on the device's current stream unless the caller names one."""
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return _serve(where, index, stream, function, *args)
    status = function(*args, torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream)
    if status != 0:
        raise LagaError(status, where)


def _empty(shape, dtype, index, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=torch.device("cuda", index))
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=torch.device("cuda", index))


def _output(shape, dtype, index, stream):
    t = _empty(shape, dtype, index, stream)
    if stream is not None:
        _kept((t,), stream)
    return t


def _int32(sh, name, t, index, stream):
    return _output(sh[name], torch.int32, index, stream) if t is None else t


def _serve_workspace(p, op, workspace, index, stream):
    """(workspace, its bytes)."""
    if workspace is None:
        workspace = _empty((max(1, laga_paged_workspace_bytes(p, op)),), torch.uint8, index, stream)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise _fault(workspace, "workspace", tuple(workspace.shape), workspace.dtype, index)
    return workspace, workspace.numel() * workspace.element_size()


def laga_page_plan(p: Paged, lengths, fresh, block_table, free_pages, free_count, lengths_out=None, free_count_out=None,
                   row_begin=None, row_request=None, position=None, slot=None, status=None, workspace=None, stream=None):
    """Pages, slots and positions of a step that adds fresh[r] tokens to request r; block_table is
    updated in place. Returns (lengths_out, free_count_out, row_begin, row_request, position, slot,
    status); lengths_out may be lengths, and free_count_out free_count. Nothing is read on the
    host: status[0] (PLAN_*) says on the device whether the step fits."""
    sh, i32, d = p.shapes(), torch.int32, _device_of(lengths, "lengths")
    lengths_out, free_count_out = _int32(sh, "lengths_out", lengths_out, d, stream), _int32(sh, "free_count_out", free_count_out, d, stream)
    row_begin, row_request = _int32(sh, "row_begin", row_begin, d, stream), _int32(sh, "row_request", row_request, d, stream)
    position, slot = _int32(sh, "position", position, d, stream), _int32(sh, "slot", slot, d, stream)
    status = _int32(sh, "status", status, d, stream)
    workspace, nbytes = _serve_workspace(p, OP_PAGE_PLAN, workspace, d, stream)
    _serve("laga_page_plan", d, stream, _lib.laga_page_plan, p.ref(), _at(lengths, "lengths", sh["lengths"], i32, d),
           _at(fresh, "fresh", sh["fresh"], i32, d), _at(block_table, "block_table", sh["block_table"], i32, d),
           _at(free_pages, "free_pages", sh["free_pages"], i32, d), _at(free_count, "free_count", (1,), i32, d),
           _at(lengths_out, "lengths_out", sh["lengths"], i32, d), _at(free_count_out, "free_count_out", (1,), i32, d),
           _at(row_begin, "row_begin", sh["row_begin"], i32, d), _at(row_request, "row_request", sh["row_request"], i32, d),
           _at(position, "position", sh["position"], i32, d), _at(slot, "slot", sh["slot"], i32, d),
           _at(status, "status", (1,), i32, d), workspace.data_ptr(), nbytes)
    return lengths_out, free_count_out, row_begin, row_request, position, slot, status


def laga_page_release(p: Paged, lengths, drop, block_table, free_pages, free_count, lengths_out=None,
                      free_count_out=None, status=None, workspace=None, stream=None):
    """The pages of the requests with drop[r] != 0 go back on the stack (free_pages is updated in
    place); returns (lengths_out, free_count_out, status)."""
    sh, i32, d = p.shapes(), torch.int32, _device_of(lengths, "lengths")
    lengths_out, free_count_out = _int32(sh, "lengths_out", lengths_out, d, stream), _int32(sh, "free_count_out", free_count_out, d, stream)
    status = _int32(sh, "status", status, d, stream)
    workspace, nbytes = _serve_workspace(p, OP_PAGE_PLAN, workspace, d, stream)
    _serve("laga_page_release", d, stream, _lib.laga_page_release, p.ref(), _at(lengths, "lengths", sh["lengths"], i32, d),
           _at(drop, "drop", sh["drop"], i32, d), _at(block_table, "block_table", sh["block_table"], i32, d),
           _at(free_pages, "free_pages", sh["free_pages"], i32, d), _at(free_count, "free_count", (1,), i32, d),
           _at(lengths_out, "lengths_out", sh["lengths"], i32, d), _at(free_count_out, "free_count_out", (1,), i32, d),
           _at(status, "status", (1,), i32, d), workspace.data_ptr(), nbytes)
    return lengths_out, free_count_out, status


def laga_cache_append(p: Paged, latent_raw, kpe_raw, position, slot, cache, gamma=None, eps=1e-6, rope_base=10000.0,
                      position_offset=0, stream=None):
    """The cache rows of new tokens, normalised latent and rotated shared key, into their slots;
    returns cache. latent_raw and kpe_raw may be columns of one wider matrix."""
    sh, dt, i32, d = p.shapes(), p.torch_dtype, torch.int32, _device_of(cache, "cache")
    lat, lat_stride = _rows_at(latent_raw, "latent_raw", sh["latent_raw"], dt, d)
    kpe, kpe_stride = _rows_at(kpe_raw, "kpe_raw", sh["kpe_raw"], dt, d)
    cfg = _CPrologue(eps, rope_base, position_offset)
    _serve("laga_cache_append", d, stream, _lib.laga_cache_append, p.ref(), ctypes.byref(cfg), lat, lat_stride,
           None if gamma is None else _at(gamma, "gamma", sh["gamma"], dt, d), kpe, kpe_stride,
           _at(position, "position", sh["position"], i32, d), _at(slot, "slot", sh["slot"], i32, d), _cache_at(p, cache, d))
    return cache


def laga_paged_attn(p: Paged, q, w_kv_b, cache, block_table, position, row_request=None, rope_base=None,
                    position_offset=0, out=None, lse=None, workspace=None, stream=None):
    """Attention of rows over the cached positions 0 .. position[t] of their requests; returns (out,
    lse). With rope_base q's rope band is turned by the row's position first (without, it has been)."""
    sh, dt, i32, d = p.shapes(), p.torch_dtype, torch.int32, _device_of(q, "q")
    if out is None:
        out = _output(sh["out"], dt, d, stream)
    if lse is None:
        lse = _output(sh["lse"], torch.float32, d, stream)
    workspace, nbytes = _serve_workspace(p, OP_PAGED_ATTN, workspace, d, stream)
    cfg = None if rope_base is None else ctypes.byref(_CPrologue(0.0, rope_base, position_offset))
    _serve("laga_paged_attn", d, stream, _lib.laga_paged_attn, p.ref(), cfg, _at(q, "q", sh["q"], dt, d),
           _at(w_kv_b, "w_kv_b", sh["w_kv_b"], dt, d), _cache_at(p, cache, d),
           _at(block_table, "block_table", sh["block_table"], i32, d),
           None if row_request is None else _at(row_request, "row_request", sh["row_request"], i32, d),
           _at(position, "position", sh["position"], i32, d), _at(out, "out", sh["out"], dt, d),
           _at(lse, "lse", sh["lse"], torch.float32, d), workspace.data_ptr(), nbytes)
    return out, lse


def _cache_q8_at(p, cache, scales, index):
    """Addresses of a pool in 8 bits and of its scales."""
    return (_cache_at(p, cache, index, torch.float8_e4m3fn), _at(scales, "scales", p.shapes()["scales"], torch.uint8, index))


def laga_cache_append_q8(p: Paged, latent_raw, kpe_raw, position, slot, cache, scales, gamma=None, eps=1e-6,
                         rope_base=10000.0, position_offset=0, stream=None):
    """laga_cache_append into a cache in 8 bits: cache [n_pages, page_size, d_c + d_rope] float8_e4m3fn, scales [n_pages,
    page_size, 2] uint8, the exponents plus 127 of the powers of two that a row's latent and shared key are multiplied by.
    Returns (cache, scales)."""
    sh, dt, i32, d = p.shapes(), p.torch_dtype, torch.int32, _device_of(cache, "cache")
    lat, lat_stride = _rows_at(latent_raw, "latent_raw", sh["latent_raw"], dt, d)
    kpe, kpe_stride = _rows_at(kpe_raw, "kpe_raw", sh["kpe_raw"], dt, d)
    cfg = _CPrologue(eps, rope_base, position_offset)
    _serve("laga_cache_append_q8", d, stream, _lib.laga_cache_append_q8, p.ref(), ctypes.byref(cfg), lat, lat_stride,
           None if gamma is None else _at(gamma, "gamma", sh["gamma"], dt, d), kpe, kpe_stride,
           _at(position, "position", sh["position"], i32, d), _at(slot, "slot", sh["slot"], i32, d),
           *_cache_q8_at(p, cache, scales, d))
    return cache, scales


def laga_cache_read_q8(p: Paged, cache, scales, block_table, position, row_request=None, c_kv=None, k_pe=None, stream=None):
    """The numbers that cached positions stand for, row t the position[t] of request row_request[t] (or t); returns (c_kv
    [rows, d_c], k_pe [rows, d_rope]) in p's element type, exactly."""
    sh, dt, i32, d = p.shapes(), p.torch_dtype, torch.int32, _device_of(cache, "cache")
    if c_kv is None:
        c_kv = _output(sh["c_kv"], dt, d, stream)
    if k_pe is None:
        k_pe = _output(sh["k_pe"], dt, d, stream)
    _serve("laga_cache_read_q8", d, stream, _lib.laga_cache_read_q8, p.ref(), *_cache_q8_at(p, cache, scales, d),
           _at(block_table, "block_table", sh["block_table"], i32, d),
           None if row_request is None else _at(row_request, "row_request", sh["row_request"], i32, d),
           _at(position, "position", sh["position"], i32, d), _at(c_kv, "c_kv", sh["c_kv"], dt, d),
           _at(k_pe, "k_pe", sh["k_pe"], dt, d))
    return c_kv, k_pe


def laga_paged_attn_q8(p: Paged, q, w_kv_b, cache, scales, block_table, position, row_request=None, rope_base=None,
                       position_offset=0, out=None, lse=None, workspace=None, stream=None):
    """laga_paged_attn on the numbers that a cache in 8 bits stands for; returns (out, lse)."""
    sh, dt, i32, d = p.shapes(), p.torch_dtype, torch.int32, _device_of(q, "q")
    if out is None:
        out = _output(sh["out"], dt, d, stream)
    if lse is None:
        lse = _output(sh["lse"], torch.float32, d, stream)
    workspace, nbytes = _serve_workspace(p, OP_PAGED_ATTN_Q8, workspace, d, stream)
    cfg = None if rope_base is None else ctypes.byref(_CPrologue(0.0, rope_base, position_offset))
    _serve("laga_paged_attn_q8", d, stream, _lib.laga_paged_attn_q8, p.ref(), cfg, _at(q, "q", sh["q"], dt, d),
           _at(w_kv_b, "w_kv_b", sh["w_kv_b"], dt, d), *_cache_q8_at(p, cache, scales, d),
           _at(block_table, "block_table", sh["block_table"], i32, d),
           None if row_request is None else _at(row_request, "row_request", sh["row_request"], i32, d),
           _at(position, "position", sh["position"], i32, d), _at(out, "out", sh["out"], dt, d),
           _at(lse, "lse", sh["lse"], torch.float32, d), workspace.data_ptr(), nbytes)
    return out, lse
