"""ctypes binding of libmas (include/mas.h); argument marshalling only.

Every step of the alignment runs in the HIP kernels of ``libmas.so``; this
module checks tensor dtypes, devices and shapes, passes raw device pointers
and the current HIP stream, and turns non-zero status codes into exceptions.
PyTorch is used only for device memory and streams.  When the library is not
built the binding raises instead of computing anything another way.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmas.so")

MAS_OK = 0
STATUS_NAMES = {0: "MAS_OK", 1: "MAS_ERR_NULL_POINTER", 2: "MAS_ERR_BAD_SHAPE", 3: "MAS_ERR_WORKSPACE", 4: "MAS_ERR_HIP",
                5: "MAS_ERR_SCRATCH", 6: "MAS_ERR_BAD_VALUE"}
STATIC_SCRATCH_BYTES = 80 << 20  # MAS_STATIC_SCRATCH_BYTES
ITEM_OK, ITEM_EMPTY, ITEM_INFEASIBLE, ITEM_OUT_OF_RANGE, ITEM_SYNC_TIMEOUT, ITEM_BAD_WORKSPACE = 0, 1, 2, 3, 4, 5

# Every function declared in include/mas.h, with its ctypes signature.
_P, _I32, _I64, _SZ, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float


class Heads(ctypes.Structure):
    """mas_heads"""

    _fields_ = [("data", _P), ("stride_b", _I64), ("stride_t", _I64), ("stride_h", _I64)]


class AttentionDesc(ctypes.Structure):
    """mas_attention_desc"""

    _fields_ = [(n, _I32) for n in ("B", "Tq", "Tk", "Hq", "Hk", "D", "dtype", "causal", "N")] + [
        ("scale", _F), ("cap", _F)] + [(n, _P) for n in ("t_q", "t_k", "slope", "doc_start", "prefix")]


class QkDesc(ctypes.Structure):
    """mas_qk_desc"""

    _fields_ = [(n, _I32) for n in ("B", "T", "Hq", "Hk", "D", "R", "P", "dtype", "interleaved")] + [
        ("eps", _F)] + [(n, _P) for n in ("wq", "wk", "cos", "sin", "pos", "t_x")]


_H, _A, _Q = ctypes.POINTER(Heads), ctypes.POINTER(AttentionDesc), ctypes.POINTER(QkDesc)
SIGNATURES = {
    "mas_workspace_bytes": ([_I32, _I32, _I32], _SZ),
    "mas_workspace_init": ([_P, _SZ, _P], ctypes.c_int),
    "mas_search": ([_P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_expand_path": ([_P, _I32, _I32, _I32, _P, _P], ctypes.c_int),
    "mas_expand_text": ([_P, _P, _I32, _I32, _I32, _I32, _I32, _P, _P], ctypes.c_int),
    "mas_loglik": ([_P, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _P, _P], ctypes.c_int),
    "mas_forward_ex": ([_P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_forward_sentinel": ([_P, _P, _P, _P, _I32, _I32, _I32, ctypes.c_float, _P, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_forward": ([_P, _P, _P, _P, _I32, _I32, _I32, _P], ctypes.c_int),
    "mas_forward_static": ([_P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P], ctypes.c_int),
    "mas_attention_workspace_bytes": ([_A, _I32], _SZ),
    "mas_attention": ([_A, _H, _H, _H, _H, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_attention_backward": ([_A, _H, _H, _H, _H, _H, _P, _H, _H, _H, _P, _SZ, _P], ctypes.c_int),
    "mas_qk_norm_rope": ([_Q, _H, _H, _H, _H, _P], ctypes.c_int),
    "mas_qk_norm_rope_workspace_bytes": ([_I32, _I32, _I32, _I32, _I32], _SZ),
    "mas_qk_norm_rope_backward": ([_Q, _H, _H, _H, _H, _H, _H, _P, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_align_loss": ([_P, _P, _P, _P, _P, _I32, _I32, _I32, _I32, _P, _P, _P, _P, _P, _SZ, _P], ctypes.c_int),
    "mas_align_loss_workspace_bytes": ([_I32, _I32, _I32, _I32], _SZ),
    "mas_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "mas_version": ([], ctypes.c_int),
}


class MasError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__(f"{fn} failed: {STATUS_NAMES.get(code, code)}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libmas.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -c \"import __graft_entry__ as g; g.build()\"` "
                "or `python paper_2409_07704_amd/build.py`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


def _check(fn: str, code: int) -> None:
    if code != MAS_OK:
        raise MasError(fn, code)


def _dev_ptr(t: torch.Tensor | None, name: str, dtype: torch.dtype, shape=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a device (cuda/hip) tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _stream(stream, device) -> int:
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on(stream, device):
    """The call's stream as a context in which to allocate: memory the call
    brings along belongs to the stream that uses it."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        raw = _stream(stream, device)
        stream = torch.cuda.ExternalStream(raw, device=device) if raw else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


def _empty(shape, dtype, device, stream):
    with _on(stream, device):
        return torch.empty(shape, dtype=dtype, device=device)


def mas_workspace_bytes(B: int, T: int, S: int) -> int:
    return int(lib().mas_workspace_bytes(B, T, S))


def mas_status_string(code: int) -> str:
    return lib().mas_status_string(code).decode()


def mas_version() -> int:
    return int(lib().mas_version())


class Workspace:
    """Device workspace for mas_search / mas_forward_ex, initialised once."""

    def __init__(self, B: int, T: int, S: int, device=None, stream=None):
        n = mas_workspace_bytes(B, T, S)
        if n == 0:
            raise ValueError(f"invalid shape B={B} T={T} S={S}")
        self.shape = (B, T, S)
        self.nbytes = n
        self._buf = _empty(n + 256, torch.uint8, device or "cuda", stream)
        off = (-self._buf.data_ptr()) % 256
        self.ptr = self._buf.data_ptr() + off
        self.device = self._buf.device
        mas_workspace_init(self.ptr, self.nbytes, stream=stream, device=self.device)

    def fits(self, B: int, T: int, S: int) -> bool:
        return mas_workspace_bytes(B, T, S) <= self.nbytes


def mas_workspace_init(ptr: int, nbytes: int, stream=None, device=None) -> None:
    _check("mas_workspace_init", lib().mas_workspace_init(ptr, nbytes, _stream(stream, device)))


def _batch(value, t_x, t_y):
    if value.dim() != 3:
        raise ValueError("value must be [B, T, S]")
    B, T, S = value.shape
    pv = _dev_ptr(value, "value", torch.float32)
    px = _dev_ptr(t_x, "t_x", torch.int32, (B,))
    py = _dev_ptr(t_y, "t_y", torch.int32, (B,))
    return B, T, S, pv, px, py


def _workspace(ws, B, T, S, device, stream):
    if ws is None:
        ws = Workspace(B, T, S, device=device, stream=stream)
    if not ws.fits(B, T, S):
        raise ValueError("workspace too small for this batch")
    return ws


def mas_search(value, t_x, t_y, row_start_out=None, score_out=None, item_status_out=None, workspace=None, stream=None,
               durations_out=None):
    """Forward pass + backtrack without the dense path; returns row_start
    [B, T+1] int32 (see mas.h).  durations_out [B, T] int32 is optional."""
    B, T, S, pv, px, py = _batch(value, t_x, t_y)
    if row_start_out is None:
        row_start_out = _empty((B, T + 1), torch.int32, value.device, stream)
    prs = _dev_ptr(row_start_out, "row_start_out", torch.int32, (B, T + 1))
    pdu = _dev_ptr(durations_out, "durations_out", torch.int32, (B, T))
    psc = _dev_ptr(score_out, "score_out", torch.float32, (B,))
    pst = _dev_ptr(item_status_out, "item_status_out", torch.int32, (B,))
    s = _stream(stream, value.device)
    ws = _workspace(workspace, B, T, S, value.device, stream)
    _check("mas_search", lib().mas_search(pv, px, py, B, T, S, prs, pdu, psc, pst, ws.ptr, ws.nbytes, s))
    return row_start_out


def mas_expand_path(row_start, S: int, path_out=None, stream=None):
    """Dense [B, T, S] uint8 path from row_start [B, T+1]."""
    if row_start.dim() != 2:
        raise ValueError("row_start must be [B, T+1]")
    B, T1 = row_start.shape
    T = T1 - 1
    prs = _dev_ptr(row_start, "row_start", torch.int32)
    if path_out is None:
        path_out = _empty((B, T, S), torch.uint8, row_start.device, stream)
    pp = _dev_ptr(path_out, "path_out", torch.uint8, (B, T, S))
    _check("mas_expand_path", lib().mas_expand_path(prs, B, T, S, pp, _stream(stream, row_start.device)))
    return path_out


def mas_expand_text(text, row_start, S: int, out=None, stream=None):
    """Aligned text grid [B, S, C] from text [B, T, C] (any 1, 2, 4 or 8-byte
    dtype) and row_start [B, T+1]: frame j copies the text row whose segment
    holds it, zeros where none does."""
    if text.dim() != 3 or row_start.dim() != 2:
        raise ValueError("text must be [B, T, C] and row_start [B, T+1]")
    B, T, C = text.shape
    prs = _dev_ptr(row_start, "row_start", torch.int32, (B, T + 1))
    pt = _dev_ptr(text, "text", text.dtype)
    if out is None:
        out = _empty((B, S, C), text.dtype, text.device, stream)
    po = _dev_ptr(out, "out", text.dtype, (B, S, C))
    _check("mas_expand_text", lib().mas_expand_text(pt, prs, B, T, S, C, text.element_size(), po,
                                                    _stream(stream, text.device)))
    return out


def mas_loglik(mu, log_sigma, z, t_x, t_y, value_out=None, stream=None):
    """Gaussian log-likelihood value [B, T, S] fp32 of frames z [B, S, D]
    under text-token Gaussians mu, log_sigma [B, T, D] (log_sigma None: unit
    variance), written for the cells of each item's feasible band only (the
    cells MAS reads); other cells of value_out are left as they are."""
    if mu.dim() != 3 or z.dim() != 3:
        raise ValueError("mu must be [B, T, D] and z [B, S, D]")
    B, T, D = mu.shape
    S = z.shape[1]
    pm = _dev_ptr(mu, "mu", torch.float32)
    pl = _dev_ptr(log_sigma, "log_sigma", torch.float32, (B, T, D))
    pz = _dev_ptr(z, "z", torch.float32, (B, S, D))
    px = _dev_ptr(t_x, "t_x", torch.int32, (B,))
    py = _dev_ptr(t_y, "t_y", torch.int32, (B,))
    if value_out is None:
        value_out = _empty((B, T, S), torch.float32, mu.device, stream)
    pv = _dev_ptr(value_out, "value_out", torch.float32, (B, T, S))
    _check("mas_loglik", lib().mas_loglik(pm, pl, pz, px, py, B, T, S, D, pv, _stream(stream, mu.device)))
    return value_out


def mas_forward_ex(value, t_x, t_y, path_out=None, score_out=None, item_status_out=None, workspace=None, stream=None):
    """Full alignment into path_out [B, T, S] uint8 with a caller workspace."""
    B, T, S, pv, px, py = _batch(value, t_x, t_y)
    if path_out is None:
        path_out = _empty((B, T, S), torch.uint8, value.device, stream)
    pp = _dev_ptr(path_out, "path_out", torch.uint8, (B, T, S))
    psc = _dev_ptr(score_out, "score_out", torch.float32, (B,))
    pst = _dev_ptr(item_status_out, "item_status_out", torch.int32, (B,))
    s = _stream(stream, value.device)
    ws = _workspace(workspace, B, T, S, value.device, stream)
    _check("mas_forward_ex", lib().mas_forward_ex(pv, px, py, pp, B, T, S, psc, pst, ws.ptr, ws.nbytes, s))
    return path_out


def mas_forward_sentinel(value, t_x, t_y, sentinel, path_out=None, score_out=None, item_status_out=None,
                         workspace=None, stream=None):
    """Full alignment in the legacy-sentinel mode: the cells Algorithm 1
    masks hold the finite negative `sentinel` (e.g. -1e9) instead of -inf."""
    B, T, S, pv, px, py = _batch(value, t_x, t_y)
    if path_out is None:
        path_out = _empty((B, T, S), torch.uint8, value.device, stream)
    pp = _dev_ptr(path_out, "path_out", torch.uint8, (B, T, S))
    psc = _dev_ptr(score_out, "score_out", torch.float32, (B,))
    pst = _dev_ptr(item_status_out, "item_status_out", torch.int32, (B,))
    s = _stream(stream, value.device)
    ws = _workspace(workspace, B, T, S, value.device, stream)
    _check("mas_forward_sentinel",
           lib().mas_forward_sentinel(pv, px, py, pp, B, T, S, float(sentinel), psc, pst, ws.ptr, ws.nbytes, s))
    return path_out


def mas_forward_static(value, t_x, t_y, path_out=None, score_out=None, item_status_out=None, stream=None):
    """Full alignment with the library's static per-device scratch as the
    workspace: allocates no device memory (see mas.h for the limit)."""
    B, T, S, pv, px, py = _batch(value, t_x, t_y)
    if path_out is None:
        path_out = _empty((B, T, S), torch.uint8, value.device, stream)
    pp = _dev_ptr(path_out, "path_out", torch.uint8, (B, T, S))
    psc = _dev_ptr(score_out, "score_out", torch.float32, (B,))
    pst = _dev_ptr(item_status_out, "item_status_out", torch.int32, (B,))
    _check("mas_forward_static", lib().mas_forward_static(pv, px, py, pp, B, T, S, psc, pst, _stream(stream, value.device)))
    return path_out


def mas_forward(value, t_x, t_y, path_out=None, stream=None):
    """Full alignment; the library allocates its workspace stream-ordered."""
    B, T, S, pv, px, py = _batch(value, t_x, t_y)
    if path_out is None:
        path_out = _empty((B, T, S), torch.uint8, value.device, stream)
    pp = _dev_ptr(path_out, "path_out", torch.uint8, (B, T, S))
    _check("mas_forward", lib().mas_forward(pv, px, py, pp, B, T, S, _stream(stream, value.device)))
    return path_out


# ------------------------------------------------ operators around the alignment
# They take tensors as data: outputs carry no gradient, whatever their inputs
# require; a caller runs the backward calls.
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _heads(t, name, like, shape):
    """mas_heads of a tensor [B, T, H, D] with contiguous channels, of the type,
    device and shape that the call's other tensors ask for."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device (cuda/hip) tensor")
    if t.dtype is not like.dtype or t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be {like.dtype if t is not like else 'float32, float16 or bfloat16'}, got {t.dtype}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must be on {like.device}, got {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    sb, st, sh, sd = t.stride()
    if sd != 1 and shape[3] > 1:
        raise ValueError(f"{name} must have contiguous channels")
    return Heads(t.data_ptr(), sb, st, sh)


def _arg(t, name, dtype, shape, like):
    """Pointer of an optional contiguous tensor on the call's device."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device (cuda/hip) tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} must be on {like.device}, got {t.device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _run_on(stream, like):
    """The call's stream as a handle."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(like.get_device())
    return _stream(stream, like.device)


def _scratch(workspace, nbytes, like, stream):
    """(pointer, bytes) of the caller's uint8 workspace, or of a new one of
    nbytes() (0 for a shape that the call will refuse), and what keeps it alive
    until the call is enqueued."""
    if workspace is not None:
        return _arg(workspace, "workspace", torch.uint8, None, like), workspace.numel(), workspace
    n = int(nbytes())
    with _on(stream, like.device):
        workspace = torch.empty(n + 256, dtype=torch.uint8, device=like.device)
    return workspace.data_ptr() + -workspace.data_ptr() % 256, n, workspace


def _attention_desc(q, k, t_q, t_k, causal, scale, cap, slope, doc_start, prefix):
    if not isinstance(q, torch.Tensor) or not isinstance(k, torch.Tensor) or q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, Tq, Hq, D] and k [B, Tk, Hk, D]")
    if not q.is_cuda:
        raise TypeError("q must be a device (cuda/hip) tensor")
    B, Tq, Hq, D = q.shape
    _, Tk, Hk, _ = k.shape
    N = 1
    if doc_start is not None:
        if doc_start.dim() != 2:
            raise ValueError("doc_start must be [B, N + 1]")
        N = doc_start.shape[1] - 1
    return AttentionDesc(B, Tq, Tk, Hq, Hk, D, _DTYPES.get(q.dtype, -1), 1 if causal else 0, N,
                         1.0 / math.sqrt(max(D, 1)) if scale is None else scale, cap,
                         _arg(t_q, "t_q", torch.int32, (B,), q), _arg(t_k, "t_k", torch.int32, (B,), q),
                         _arg(slope, "slope", torch.float32, (Hq,), q),
                         _arg(doc_start, "doc_start", torch.int32, (B, N + 1), q),
                         _arg(prefix, "prefix", torch.int32, (B, N), q)), (B, Tk, Hk, D)


def mas_attention_workspace_bytes(q, k, backward: bool = False) -> int:
    """Bytes of workspace for mas_attention of q [B, Tq, Hq, D] over k [B, Tk,
    Hk, D] and, with `backward`, for mas_attention_backward too."""
    d, _ = _attention_desc(q, k, None, None, False, None, 0.0, None, None, None)
    return int(lib().mas_attention_workspace_bytes(d, 1 if backward else 0))


def mas_attention(q, k, v, t_q=None, t_k=None, causal=False, scale=None, cap=0.0, slope=None, doc_start=None,
                  prefix=None, out=None, lse_out=None, workspace=None, stream=None):
    """Attention of q [B, Tq, Hq, D] over k, v [B, Tk, Hk, D] (any strides,
    channels contiguous); returns out [B, Tq, Hq, D].

    scale None: 1 / sqrt(D).  cap > 0: scores become cap * tanh(score / cap).
    slope [Hq] fp32: minus slope * distance.  t_q, t_k [B] int32: lengths; the
    queries are the last t_q tokens of the t_k.  causal, doc_start [B, N + 1]
    and prefix [B, N] int32: see mas.h.  lse_out [B, Hq, Tq] fp32 is what the
    backward pass takes.  workspace: a uint8 tensor of
    mas_attention_workspace_bytes, 256-byte aligned, or None.  Not recorded
    by autograd: mas_attention_backward computes the gradients."""
    d, kv = _attention_desc(q, k, t_q, t_k, causal, scale, cap, slope, doc_start, prefix)
    hq, hk, hv = _heads(q, "q", q, q.shape), _heads(k, "k", q, kv), _heads(v, "v", q, kv)
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    ho = _heads(out, "out", q, q.shape)
    pl = _arg(lse_out, "lse_out", torch.float32, (d.B, d.Hq, d.Tq), q)
    L = lib()
    ws, n, keep = _scratch(workspace, lambda: L.mas_attention_workspace_bytes(d, 0), q, stream)
    _check("mas_attention", L.mas_attention(d, hq, hk, hv, ho, pl, ws, n, _run_on(stream, q)))
    return out


def mas_attention_backward(dout, q, k, v, out, lse, t_q=None, t_k=None, causal=False, scale=None, cap=0.0, slope=None,
                           doc_start=None, prefix=None, dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Gradients (dq, dk, dv) of mas_attention from dout [B, Tq, Hq, D], the
    inputs, and the forward call's out and lse_out; other arguments as there."""
    d, kv = _attention_desc(q, k, t_q, t_k, causal, scale, cap, slope, doc_start, prefix)
    hq, hk, hv = _heads(q, "q", q, q.shape), _heads(k, "k", q, kv), _heads(v, "v", q, kv)
    ho, hg = _heads(out, "out", q, q.shape), _heads(dout, "dout", q, q.shape)
    if lse is None:
        raise TypeError("lse must be a device (cuda/hip) tensor")
    pl = _arg(lse, "lse", torch.float32, (d.B, d.Hq, d.Tq), q)
    dq = _empty(q.shape, q.dtype, q.device, stream) if dq is None else dq
    dk = _empty(kv, q.dtype, q.device, stream) if dk is None else dk
    dv = _empty(kv, q.dtype, q.device, stream) if dv is None else dv
    gq, gk, gv = _heads(dq, "dq", q, q.shape), _heads(dk, "dk", q, kv), _heads(dv, "dv", q, kv)
    L = lib()
    ws, n, keep = _scratch(workspace, lambda: L.mas_attention_workspace_bytes(d, 1), q, stream)
    _check("mas_attention_backward",
           L.mas_attention_backward(d, hg, hq, hk, hv, ho, pl, gq, gk, gv, ws, n, _run_on(stream, q)))
    return dq, dk, dv


def _qk_desc(q, k, wq, wk, cos, sin, pos, t_x, eps, interleaved):
    if not isinstance(q, torch.Tensor) or q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q must be [B, T, Hq, D] and k [B, T, Hk, D] or None")
    if not q.is_cuda:
        raise TypeError("q must be a device (cuda/hip) tensor")
    B, T, Hq, D = q.shape
    Hk = 0 if k is None else k.shape[2]
    if (cos is None) != (sin is None) or (cos is not None and cos.dim() != 2):
        raise ValueError("cos and sin must both be [P, R / 2], or None")
    P, half = (0, 0) if cos is None else cos.shape
    return QkDesc(B, T, Hq, Hk, D, 2 * half, P, _DTYPES.get(q.dtype, -1), 1 if interleaved else 0, eps,
                  _arg(wq, "wq", torch.float32, (D,), q), _arg(wk, "wk", torch.float32, (D,), q),
                  _arg(cos, "cos", torch.float32, (P, half), q), _arg(sin, "sin", torch.float32, (P, half), q),
                  _arg(pos, "pos", torch.int32, (B, T), q), _arg(t_x, "t_x", torch.int32, (B,), q)), (B, T, Hk, D)


def mas_qk_norm_rope(q, k, wq, wk, cos, sin, pos=None, t_x=None, eps=1e-6, interleaved=False, q_out=None, k_out=None,
                     stream=None):
    """Norm of q [B, T, Hq, D] and k [B, T, Hk, D] (k may be None) for each
    head, weighted by wq, wk [D] fp32 (None: 1), and the rotation of the first
    R channels by the rows pos [B, T] int32 (None: the token's index) of cos,
    sin [P, R / 2] fp32; returns (q_out, k_out).  Padding (t >= t_x) becomes
    zeros.  q_out, k_out may be q, k.  Not recorded by autograd:
    mas_qk_norm_rope_backward computes the gradients."""
    d, ks = _qk_desc(q, k, wq, wk, cos, sin, pos, t_x, eps, interleaved)
    hq, hk = _heads(q, "q", q, q.shape), None if k is None else _heads(k, "k", q, ks)
    q_out = _empty(q.shape, q.dtype, q.device, stream) if q_out is None else q_out
    if k is None:
        k_out = None
    elif k_out is None:
        k_out = _empty(ks, q.dtype, q.device, stream)
    oq, ok = _heads(q_out, "q_out", q, q.shape), None if k is None else _heads(k_out, "k_out", q, ks)
    _check("mas_qk_norm_rope", lib().mas_qk_norm_rope(d, hq, hk, oq, ok, _run_on(stream, q)))
    return q_out, k_out


def mas_qk_norm_rope_workspace_bytes(q, k) -> int:
    """Bytes of workspace for mas_qk_norm_rope_backward."""
    B, T, Hq, D = q.shape
    return int(lib().mas_qk_norm_rope_workspace_bytes(B, T, Hq, 0 if k is None else k.shape[2], D))


def mas_qk_norm_rope_backward(dq_out, dk_out, q, k, wq, wk, cos, sin, pos=None, t_x=None, eps=1e-6, interleaved=False,
                              dq=None, dk=None, dwq=None, dwk=None, workspace=None, stream=None):
    """Gradients (dq, dk, dwq, dwk) of mas_qk_norm_rope from those of its
    outputs and its inputs; dwq, dwk [D] fp32.  dk, dwk are None without k."""
    d, ks = _qk_desc(q, k, wq, wk, cos, sin, pos, t_x, eps, interleaved)
    hq, hk = _heads(q, "q", q, q.shape), None if k is None else _heads(k, "k", q, ks)
    gq, gk = _heads(dq_out, "dq_out", q, q.shape), None if k is None else _heads(dk_out, "dk_out", q, ks)
    dq = _empty(q.shape, q.dtype, q.device, stream) if dq is None else dq
    dwq = _empty((d.D,), torch.float32, q.device, stream) if dwq is None else dwq
    if k is None:
        dk = dwk = None
    else:
        dk = _empty(ks, q.dtype, q.device, stream) if dk is None else dk
        dwk = _empty((d.D,), torch.float32, q.device, stream) if dwk is None else dwk
    oq, ok = _heads(dq, "dq", q, q.shape), None if k is None else _heads(dk, "dk", q, ks)
    pq, pk = _arg(dwq, "dwq", torch.float32, (d.D,), q), _arg(dwk, "dwk", torch.float32, (d.D,), q)
    L = lib()
    ws, n, keep = _scratch(workspace, lambda: L.mas_qk_norm_rope_workspace_bytes(d.B, d.T, d.Hq, d.Hk, d.D), q, stream)
    _check("mas_qk_norm_rope_backward",
           L.mas_qk_norm_rope_backward(d, gq, gk, hq, hk, oq, ok, pq, pk, ws, n, _run_on(stream, q)))
    return dq, dk, dwq, dwk


def mas_align_loss_workspace_bytes(B: int, T: int, S: int, D: int) -> int:
    return int(lib().mas_align_loss_workspace_bytes(B, T, S, D))


def mas_align_loss(mu, log_sigma, z, row_start, item_weight=None, loss_out=None, dmu=None, dlog_sigma=None, dz=None,
                   workspace=None, stream=None, gradients=True):
    """Negative log-likelihood [B] of the frames z [B, S, D] under the rows of
    mu, log_sigma [B, T, D] (log_sigma None: unit variance) that row_start [B,
    T + 1] gives them, and the gradients of the items' losses, each times
    item_weight [B] (None: 1); returns (loss, dmu, dlog_sigma, dz).  dlog_sigma
    is None without log_sigma unless given; without `gradients` only those given
    are made.  Not recorded by autograd."""
    if not isinstance(mu, torch.Tensor) or mu.dim() != 3 or z.dim() != 3:
        raise ValueError("mu must be [B, T, D] and z [B, S, D]")
    B, T, D = mu.shape
    S, f32 = z.shape[1], torch.float32
    pm, pl = _arg(mu, "mu", f32, mu.shape, mu), _arg(log_sigma, "log_sigma", f32, mu.shape, mu)
    pz = _arg(z, "z", f32, (B, S, D), mu)
    pr = _arg(row_start, "row_start", torch.int32, (B, T + 1), mu)
    pw = _arg(item_weight, "item_weight", f32, (B,), mu)
    if pz is None or pr is None:
        raise TypeError("z and row_start must be device (cuda/hip) tensors")
    loss_out = _empty((B,), f32, mu.device, stream) if loss_out is None else loss_out
    if gradients:
        dmu = _empty((B, T, D), f32, mu.device, stream) if dmu is None else dmu
        dz = _empty((B, S, D), f32, mu.device, stream) if dz is None else dz
        if dlog_sigma is None and log_sigma is not None:
            dlog_sigma = _empty((B, T, D), f32, mu.device, stream)
    po = _arg(loss_out, "loss_out", f32, (B,), mu)
    gm, gl = _arg(dmu, "dmu", f32, mu.shape, mu), _arg(dlog_sigma, "dlog_sigma", f32, mu.shape, mu)
    gz = _arg(dz, "dz", f32, (B, S, D), mu)
    L = lib()
    ws, n, keep = _scratch(workspace, lambda: L.mas_align_loss_workspace_bytes(B, T, S, D), mu, stream)
    _check("mas_align_loss", L.mas_align_loss(pm, pl, pz, pr, pw, B, T, S, D, po, gm, gl, gz, ws, n, _run_on(stream, mu)))
    return loss_out, dmu, dlog_sigma, dz
