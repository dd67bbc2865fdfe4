"""Operators around the collectives, for torch tensors on one GPU: a thin
layer over the C ABI in include/ar_ops.h (formulas and roundings there).

    gated_ffn, gated_ffn_backward           act(x Wg^T) * (x Wu^T)
    residual_norm, residual_norm_backward   norm, gate, scaled residual, norm
    orthogonalize                           Newton-Schulz steps on an update
    packed_attention, packed_attention_backward
                                            attention over packed sequences
    vocab_loss, vocab_loss_part, vocab_loss_join, vocab_loss_backward
                                            cross entropy over a vocabulary

Every step runs in the HIP library; torch provides device memory and streams.
Tensors are checked on every call (ValueError, TypeError); what the library
itself refuses is an ARError.  Results and workspaces are allocated by torch
on the stream of the call (``stream``, or torch's current one); a result given
as ``out`` is written in place.  Rows must be contiguous; the stride between
rows is free.

Results have no autograd graph, whatever the arguments require: gradients come
from the *_backward functions.  The first call with a tensor that requires one,
outside of torch.no_grad(), warns (RuntimeWarning).

Calls on the current stream that make their own results are checked and made in
native code (csrc/ops_args.cpp, used with the torch it was built against); what
is not plainly right there, and every other call, takes the checks below.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import paper_2603_11438_amd as _ar

OPS_ARGS_PATH = os.path.join(os.path.dirname(_ar.LIB_PATH), "_ops_args.so")

AR_NORM_POST, AR_NORM_PRE = 1, 2
AR_ACT_SILU, AR_ACT_GELU, AR_ACT_RELU = 0, 1, 2
AR_ORTHO_MAX_STEPS = 16
AR_ATTN_CAUSAL, AR_ATTN_CLEAR = 1, 2
ACTS = {"silu": AR_ACT_SILU, "gelu": AR_ACT_GELU, "relu": AR_ACT_RELU}

_P, _S, _I, _F = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float


class ar_norm_desc(ctypes.Structure):
    _fields_ = [("rows", _S), ("cols", _S), ("dtype", _I), ("param_dtype", _I), ("flags", _I), ("alpha", _F),
                ("eps", _F), ("gate_rows", _S), ("ld_y", _S), ("ld_residual", _S), ("ld_s", _S), ("ld_x", _S),
                ("ld_ds", _S), ("ld_dx", _S), ("ld_dy", _S)]


class ar_ffn_desc(ctypes.Structure):
    _fields_ = [("tokens", _S), ("dim", _S), ("hidden", _S), ("dtype", _I), ("act", _I), ("ld_x", _S),
                ("ld_w_gate", _S), ("ld_w_up", _S), ("ld_h", _S), ("ld_dx", _S), ("ld_dw_gate", _S), ("ld_dw_up", _S)]


class ar_ortho_desc(ctypes.Structure):
    _fields_ = [("batch", _S), ("rows", _S), ("cols", _S), ("dtype", _I), ("steps", _I), ("coefs", ctypes.POINTER(_F)),
                ("eps", _F), ("scale", _F), ("ld_in", _S), ("ld_out", _S), ("stride_in", _S), ("stride_out", _S)]


class ar_attention_desc(ctypes.Structure):
    _fields_ = [("sequences", _S), ("tokens_q", _S), ("tokens_k", _S), ("heads", _S), ("kv_heads", _S), ("dim", _S), ("dtype", _I),
                ("flags", _I), ("scale", _F)] + [(kind + name, _S) for name in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")
                                                 for kind in ("ld_", "hs_")]


class ar_vocab_desc(ctypes.Structure):
    _fields_ = [("tokens", _S), ("dim", _S), ("rows", _S), ("first", _S), ("classes", _S), ("dtype", _I), ("target_bytes", _I),
                ("ld_x", _S), ("ld_w", _S), ("ld_dx", _S), ("ld_dw", _S)]


# Every symbol include/ar_ops.h declares, with (restype, argtypes).
SIGNATURES = {
    "ar_residual_norm": (_I, [ctypes.POINTER(ar_norm_desc)] + [_P] * 8),
    "ar_residual_norm_backward": (_I, [ctypes.POINTER(ar_norm_desc)] + [_P] * 13 + [_S, _P]),
    "ar_residual_norm_backward_workspace": (_S, [ctypes.POINTER(ar_norm_desc)]),
    "ar_gated_ffn": (_I, [ctypes.POINTER(ar_ffn_desc)] + [_P] * 6 + [_S, _P]),
    "ar_gated_ffn_workspace": (_S, [ctypes.POINTER(ar_ffn_desc)]),
    "ar_gated_ffn_workspace_for": (_S, [ctypes.POINTER(ar_ffn_desc)] + [_P] * 3),
    "ar_gated_ffn_backward": (_I, [ctypes.POINTER(ar_ffn_desc)] + [_P] * 9 + [_S, _P]),
    "ar_gated_ffn_backward_workspace": (_S, [ctypes.POINTER(ar_ffn_desc)]),
    "ar_orthogonalize": (_I, [ctypes.POINTER(ar_ortho_desc)] + [_P] * 3 + [_S, _P]),
    "ar_orthogonalize_workspace": (_S, [ctypes.POINTER(ar_ortho_desc)]),
    "ar_attention": (_I, [ctypes.POINTER(ar_attention_desc)] + [_P] * 8 + [_S, _P]),
    "ar_attention_workspace": (_S, [ctypes.POINTER(ar_attention_desc)]),
    "ar_attention_workspace_for": (_S, [ctypes.POINTER(ar_attention_desc)] + [_P] * 3),
    "ar_attention_backward": (_I, [ctypes.POINTER(ar_attention_desc)] + [_P] * 12 + [_S, _P]),
    "ar_attention_backward_workspace": (_S, [ctypes.POINTER(ar_attention_desc)]),
    "ar_vocab_loss": (_I, [ctypes.POINTER(ar_vocab_desc)] + [_P] * 6 + [_S, _P]),
    "ar_vocab_loss_workspace": (_S, [ctypes.POINTER(ar_vocab_desc), _P, _P]),
    "ar_vocab_loss_part": (_I, [ctypes.POINTER(ar_vocab_desc)] + [_P] * 5 + [_S, _P]),
    "ar_vocab_loss_join": (_I, [ctypes.POINTER(ar_vocab_desc), _S] + [_P] * 5),
    "ar_vocab_loss_backward": (_I, [ctypes.POINTER(ar_vocab_desc), _P, _S] + [_P] * 7 + [_S, _P]),
    "ar_vocab_loss_backward_workspace": (_S, [ctypes.POINTER(ar_vocab_desc), _P, _P, _I, _I]),
}

_bound = None


def _lib() -> ctypes.CDLL:
    global _bound
    if _bound is None:
        L = _ar.lib()
        for name, (res, args) in SIGNATURES.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _bound = L
    return _bound


class _Native:
    """The native call path and the addresses of the functions it calls."""

    def __init__(self):
        import importlib.util

        import torch  # the extension's symbols come from torch's libraries

        if not os.path.exists(OPS_ARGS_PATH):
            raise ImportError(f"not built ({OPS_ARGS_PATH} missing); run __graft_entry__.build()")
        spec = importlib.util.spec_from_file_location("_ops_args", OPS_ARGS_PATH)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        if mod.torch_version != str(torch.__version__):
            # it reads torch's C++ objects as that version laid them out
            raise ImportError(f"built against torch {mod.torch_version}, loaded is {torch.__version__}")
        L = _lib()
        address = lambda name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value  # noqa: E731
        self.tell_graphs = mod.tell_graphs
        self.tell_graphs(_graphs_told)
        self.norm, self.norm_backward, self.ffn, self.ffn_backward = mod.norm, mod.norm_backward, mod.ffn, mod.ffn_backward
        self.norm_fn = address("ar_residual_norm")
        self.norm_backward_fns = address("ar_residual_norm_backward"), address("ar_residual_norm_backward_workspace")
        self.ffn_fns = address("ar_gated_ffn"), address("ar_gated_ffn_workspace_for")
        self.ffn_backward_fns = address("ar_gated_ffn_backward"), address("ar_gated_ffn_backward_workspace")
        self.attention, self.vocab_loss = mod.attention, mod.vocab_loss
        self.attention_fns = address("ar_attention"), address("ar_attention_workspace_for")
        self.vocab_loss_fns = address("ar_vocab_loss"), address("ar_vocab_loss_workspace")
        self.in_use, self.device, self.stream = torch.cuda.is_initialized, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


_native_path = None  # not looked for yet; False: cannot be used


def _native() -> Optional[_Native]:
    """The native call path, where there is a device context to call it in; None
    (with a warning, once) where it cannot be used."""
    global _native_path
    if _native_path is None:
        try:
            _native_path = _Native()
        except (ImportError, AttributeError) as e:  # AttributeError: a torch without devices
            import warnings

            warnings.warn(f"the native part of the operators' binding cannot be used: {e}; tensors are checked in Python, "
                          "some 10 us per call", RuntimeWarning, stacklevel=3)
            _native_path = False
    return _native_path if _native_path and _native_path.in_use() else None


_graphs_told = False


def _tell_of_graphs(*tensors):
    """Warns, once, where autograd would expect a graph that results do not have."""
    global _graphs_told
    if _graphs_told:
        return
    import torch

    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        import warnings

        _graphs_told = True
        if (nat := _native()) is not None:
            nat.tell_graphs(True)
        warnings.warn("the results of this package's operators have no autograd graph: gradients come from the *_backward functions "
                      "(torch.no_grad() or detached tensors say that this is known)", RuntimeWarning, stacklevel=3)


def _done(got, what):
    """The results of a native call; raises for a status."""
    if type(got) is int:
        _ar._check(got, what)
    return got


# ---- tensors ----------------------------------------------------------------

class _On:
    """The device and stream of a call: makes them current where they are not,
    so that what torch allocates belongs to the call's stream."""

    def __init__(self, t, stream):
        import torch

        if not t.is_cuda:
            raise ValueError("tensors must be on the GPU")
        self.index = t.device.index
        if stream is not None and stream.device.index != self.index:
            raise ValueError(f"the stream is on {stream.device}, the tensors are on {t.device}")
        self.guard = None
        if stream is not None:
            self.guard = torch.cuda.stream(stream)
        elif torch._C._cuda_getDevice() != self.index:
            self.guard = torch.cuda.device(self.index)

    def __enter__(self):
        import torch

        if self.guard is not None:
            self.guard.__enter__()
        self.ptr = torch._C._cuda_getCurrentRawStream(self.index)
        return self

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _rows(t, name, cols=None, rows=None, dtype=None, device=None):
    """(rows, cols, row stride) of a tensor whose leading dimensions count rows."""
    if not t.is_cuda or (device is not None and t.device.index != device):
        raise ValueError(f"{name} must be on the GPU of the call")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    n, stride = shape[-1], t.stride()
    m = 1
    for k in shape[:-1]:
        m *= k
    if (cols is not None and n != cols) or (rows is not None and m != rows):
        raise ValueError(f"{name} is {m} x {n}, expected {m if rows is None else rows} x {n if cols is None else cols}")
    if m == 0 or n == 0:
        return m, n, n
    if n > 1 and stride[-1] != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    ld, span = n, None
    for k, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if k == 1:
            continue
        if span is None:
            ld = s
        elif s != span:
            raise ValueError(f"the leading dimensions of {name} must have one stride between rows")
        span = s * k
    if ld < n:
        raise ValueError(f"the rows of {name} must not overlap")
    return m, n, ld


def _param(t, name, shape, dtype, device):
    if t is None:
        return None
    if not t.is_cuda or t.device.index != device or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name} must be a contiguous tensor of shape {shape} on the GPU of the call")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    return t.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _workspace(nbytes, like):
    import torch

    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


# ---- residual norm ------------------------------------------------------------

def _norm_desc(y, post_weight, pre_weight, gate, alpha, eps, post, pre):
    """Description, and the pointers of the parameters (post, gate, pre)."""
    import torch

    rows, cols, ld = _rows(y, "y")
    dev = y.device.index
    given = [t for t in (post_weight, gate, pre_weight) if t is not None]
    pdt = given[0].dtype if given else y.dtype
    d = ar_norm_desc(rows=rows, cols=cols, dtype=_ar._dtype_of(y), param_dtype=_ar.AR_FLOAT32 if pdt == torch.float32 else
                     _ar.AR_BFLOAT16, flags=(AR_NORM_POST if post else 0) | (AR_NORM_PRE if pre else 0), alpha=alpha,
                     eps=eps, gate_rows=0, ld_y=ld)
    if pdt not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported dtype {pdt}")
    if gate is not None:
        if gate.dim() not in (1, 2):
            raise ValueError("gate must be a row or a matrix")
        d.gate_rows = 1 if gate.dim() == 1 else gate.shape[0]
        if d.gate_rows == 0 or rows % d.gate_rows:
            raise ValueError(f"{rows} rows cannot be shared by {d.gate_rows} rows of the gate")
    if (post_weight is not None and not post) or (pre_weight is not None and not pre):
        raise ValueError("a weight is given for a norm that is switched off")
    gshape = None if gate is None else ((cols,) if gate.dim() == 1 else (d.gate_rows, cols))
    return d, pdt, (_param(post_weight, "post_weight", (cols,), pdt, dev), _param(gate, "gate", gshape, pdt, dev),
                    _param(pre_weight, "pre_weight", (cols,), pdt, dev))


def residual_norm(y, residual, *, post_weight=None, pre_weight=None, gate=None, alpha: float = 1.0, eps: float = 1e-6,
                  post: bool = True, pre: bool = True, out=None, stream=None):
    """s = alpha * residual + gate * norm(y), x = norm(s); returns (s, x).

    y and residual: (..., cols), f32 or bf16.  Weights (cols) and gate (cols, or
    (k, cols) with row i for the i-th rows / k consecutive rows) share one type
    of their own; one left out is ones.  post / pre switch the norm of y and
    the norm of s off; without the latter x is None.  out: (s, x) to write to;
    s may be y or residual, and so may x."""
    import torch

    if out is None and stream is None and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.norm(nat.norm_fn, y, residual, post_weight, pre_weight, gate, alpha, eps,
                       (AR_NORM_POST if post else 0) | (AR_NORM_PRE if pre else 0), dev, nat.stream(dev))
        if got is not None:
            return _done(got, "ar_residual_norm")
    _tell_of_graphs(y, residual, post_weight, pre_weight, gate)
    with _On(y, stream) as on:
        d, _, (w1, g, w2) = _norm_desc(y, post_weight, pre_weight, gate, alpha, eps, post, pre)
        dev = on.index
        _, _, d.ld_residual = _rows(residual, "residual", d.cols, d.rows, y.dtype, dev)
        if out is None:
            s, x = torch.empty_like(y, memory_format=torch.contiguous_format), None
            if pre:
                x = torch.empty_like(s)
        else:
            s, x = out
            if (x is None) == pre:
                raise ValueError("out is (s, x), x None where the norm of s is switched off")
        _, _, d.ld_s = _rows(s, "s", d.cols, d.rows, y.dtype, dev)
        if x is not None:
            _, _, d.ld_x = _rows(x, "x", d.cols, d.rows, y.dtype, dev)
        rc = _lib().ar_residual_norm(ctypes.byref(d), y.data_ptr(), residual.data_ptr(), w1, g, w2, s.data_ptr(), _ptr(x),
                                     on.ptr)
        _ar._check(rc, "ar_residual_norm")
    return s, x


def residual_norm_backward(y, s, ds, dx, *, post_weight=None, pre_weight=None, gate=None, alpha: float = 1.0,
                           eps: float = 1e-6, post: bool = True, pre: bool = True, param_grads: bool = True, out=None,
                           workspace=None, stream=None) -> dict:
    """Gradients of residual_norm: {"dy", "dresidual", "dpost_weight",
    "dpre_weight", "dgate"}; those of parameters that are absent, or not wanted
    (param_grads False), are left out.

    y: as in the forward call, s: its result; ds (None = zero) and dx (None
    where x was not computed): the gradients of s and x.  out: (dy, dresidual)
    to write to; each may be y, s, ds or dx.  workspace: a uint8 tensor to use
    in place of a new one (residual_norm_backward_workspace)."""
    import torch

    if out is None and workspace is None and stream is None and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.norm_backward(*nat.norm_backward_fns, y, s, ds, dx, post_weight, pre_weight, gate, alpha, eps,
                                (AR_NORM_POST if post else 0) | (AR_NORM_PRE if pre else 0), param_grads, dev, nat.stream(dev))
        if got is not None:
            got = zip(("dy", "dresidual", "dpost_weight", "dpre_weight", "dgate"), _done(got, "ar_residual_norm_backward"))
            return {k: t for k, t in got if t is not None}
    _tell_of_graphs(y, s, ds, dx, post_weight, pre_weight, gate)
    with _On(y, stream) as on:
        d, pdt, (w1, g, w2) = _norm_desc(y, post_weight, pre_weight, gate, alpha, eps, post, pre)
        dev = on.index
        _, _, d.ld_s = _rows(s, "s", d.cols, d.rows, y.dtype, dev)
        if ds is not None:
            _, _, d.ld_ds = _rows(ds, "ds", d.cols, d.rows, y.dtype, dev)
        if (dx is not None) != pre:
            raise ValueError("dx is given exactly where the norm of s is not switched off")
        if pre:
            _, _, d.ld_dx = _rows(dx, "dx", d.cols, d.rows, y.dtype, dev)
        if out is None:
            dy = torch.empty_like(y, memory_format=torch.contiguous_format)
            dr = torch.empty_like(dy)
        else:
            dy, dr = out
        _, _, d.ld_dy = _rows(dy, "dy", d.cols, d.rows, y.dtype, dev)
        _, _, d.ld_residual = _rows(dr, "dresidual", d.cols, d.rows, y.dtype, dev)
        grads = {"dy": dy, "dresidual": dr}
        if param_grads:
            for key, t in (("dpost_weight", post_weight), ("dpre_weight", pre_weight), ("dgate", gate)):
                if t is not None:
                    grads[key] = torch.empty_like(t)
        ws = workspace
        need = _lib().ar_residual_norm_backward_workspace(ctypes.byref(d)) if len(grads) > 2 else 0
        if ws is None:
            ws = _workspace(need, y)
        elif not ws.is_cuda or ws.device.index != dev or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU of the call")
        rc = _lib().ar_residual_norm_backward(
            ctypes.byref(d), y.data_ptr(), s.data_ptr(), _ptr(ds), _ptr(dx), w1, g, w2, dy.data_ptr(), dr.data_ptr(),
            _ptr(grads.get("dpost_weight")), _ptr(grads.get("dgate")), _ptr(grads.get("dpre_weight")), _ptr(ws),
            0 if ws is None else ws.numel() * ws.element_size(), on.ptr)
        _ar._check(rc, "ar_residual_norm_backward")
    return grads


def residual_norm_backward_workspace(rows: int, cols: int, dtype="f32") -> int:
    """Bytes of residual_norm_backward's workspace."""
    d = ar_norm_desc(rows=rows, cols=cols, dtype=_ar.DTYPES[dtype], param_dtype=0, flags=3, alpha=1.0, eps=1.0)
    return _lib().ar_residual_norm_backward_workspace(ctypes.byref(d))


# ---- gated feed-forward block -------------------------------------------------

def _ffn_desc(x, w_gate, w_up, act):
    if act not in ACTS:
        raise ValueError(f"unknown activation {act!r}: one of {sorted(ACTS)}")
    tokens, dim, ld_x = _rows(x, "x")
    dev = x.device.index
    if w_gate.dim() != 2 or w_up.dim() != 2:
        raise ValueError("the weights must be matrices")
    hidden, _, ld_g = _rows(w_gate, "w_gate", dim, None, x.dtype, dev)
    _, _, ld_u = _rows(w_up, "w_up", dim, hidden, x.dtype, dev)
    return ar_ffn_desc(tokens=tokens, dim=dim, hidden=hidden, dtype=_ar._dtype_of(x), act=ACTS[act], ld_x=ld_x,
                       ld_w_gate=ld_g, ld_w_up=ld_u)


def gated_ffn(x, w_gate, w_up, *, act: str = "silu", save: bool = False, out=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T), bf16; with save also what
    gated_ffn_backward needs: (h, saved).

    x: (..., dim); weights: (hidden, dim), which may be halves of one tensor;
    act: "silu", "gelu" (the form with tanh) or "relu"; out: h to write to.
    saved: (2, tokens, hidden) fp32, both projections."""
    import torch

    if out is None and stream is None and act in ACTS and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.ffn(*nat.ffn_fns, x, w_gate, w_up, ACTS[act], save, dev, nat.stream(dev))
        if got is not None:
            h, saved = _done(got, "ar_gated_ffn")
            return (h, saved) if save else h
    _tell_of_graphs(x, w_gate, w_up)
    with _On(x, stream) as on:
        d = _ffn_desc(x, w_gate, w_up, act)
        h = out
        if h is None:
            h = torch.empty(*x.shape[:-1], d.hidden, dtype=x.dtype, device=x.device)
        _, _, d.ld_h = _rows(h, "h", d.hidden, d.tokens, x.dtype, on.index)
        saved = torch.empty(2, d.tokens, d.hidden, dtype=torch.float32, device=x.device) if save else None
        L = _lib()
        # only operands that have to be laid out, and a dim in several runs, need one
        need = L.ar_gated_ffn_workspace_for(ctypes.byref(d), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr())
        ws = _workspace(need, x)
        rc = L.ar_gated_ffn(ctypes.byref(d), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), h.data_ptr(), _ptr(saved),
                            _ptr(ws), need, on.ptr)
        _ar._check(rc, "ar_gated_ffn")
    return (h, saved) if save else h


def gated_ffn_backward(dh, x, w_gate, w_up, saved, *, act: str = "silu", need_dx: bool = True, need_dw: bool = True,
                       out=None, workspace=None, stream=None):
    """Gradients of gated_ffn with regard to x and both weights: (dx, dw_gate,
    dw_up); None for those not needed (need_dx, need_dw).

    saved: from gated_ffn(save=True) on the same x and weights.  out: the three
    results to write to.  workspace: a uint8 tensor to use in place of a new one
    (gated_ffn_backward_workspace)."""
    import torch

    if out is None and workspace is None and stream is None and act in ACTS and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.ffn_backward(*nat.ffn_backward_fns, dh, x, w_gate, w_up, saved, ACTS[act], need_dx, need_dw, dev, nat.stream(dev))
        if got is not None:
            return _done(got, "ar_gated_ffn_backward")
    _tell_of_graphs(dh, x, w_gate, w_up)
    with _On(x, stream) as on:
        d = _ffn_desc(x, w_gate, w_up, act)
        dev = on.index
        _, _, d.ld_h = _rows(dh, "dh", d.hidden, d.tokens, x.dtype, dev)
        if (not saved.is_cuda or saved.device.index != dev or saved.dtype != torch.float32 or not saved.is_contiguous()
                or tuple(saved.shape) != (2, d.tokens, d.hidden)):
            raise ValueError("saved must be what gated_ffn(save=True) returned for this x and these weights")
        dx, dg, du = (None, None, None) if out is None else out
        if need_dx:
            dx = torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx
            _, _, d.ld_dx = _rows(dx, "dx", d.dim, d.tokens, x.dtype, dev)
        if need_dw:
            dg = torch.empty(d.hidden, d.dim, dtype=x.dtype, device=x.device) if dg is None else dg
            du = torch.empty_like(dg, memory_format=torch.contiguous_format) if du is None else du
            _, _, d.ld_dw_gate = _rows(dg, "dw_gate", d.dim, d.hidden, x.dtype, dev)
            _, _, d.ld_dw_up = _rows(du, "dw_up", d.dim, d.hidden, x.dtype, dev)
        L, ws = _lib(), workspace
        if ws is None:
            ws = _workspace(L.ar_gated_ffn_backward_workspace(ctypes.byref(d)), x)
        elif not ws.is_cuda or ws.device.index != dev or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU of the call")
        rc = L.ar_gated_ffn_backward(
            ctypes.byref(d), dh.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), saved.data_ptr(),
            _ptr(dx) if need_dx else None, _ptr(dg) if need_dw else None, _ptr(du) if need_dw else None, _ptr(ws),
            0 if ws is None else ws.numel() * ws.element_size(), on.ptr)
        _ar._check(rc, "ar_gated_ffn_backward")
    return dx if need_dx else None, dg if need_dw else None, du if need_dw else None


def gated_ffn_backward_workspace(tokens: int, dim: int, hidden: int) -> int:
    """Bytes of gated_ffn_backward's workspace."""
    d = ar_ffn_desc(tokens=tokens, dim=dim, hidden=hidden, dtype=_ar.AR_BFLOAT16)
    return _lib().ar_gated_ffn_backward_workspace(ctypes.byref(d))


# ---- orthogonalised updates ---------------------------------------------------

#: Coefficients (a, b, c) of a step that takes singular values in (0, 1] near 1
#: within five steps.
ORTHO_COEFS = (3.4445, -4.7750, 2.0315)


def _matrices(t, name):
    """(batch, rows, cols, row stride, stride between matrices)."""
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be a matrix or a batch of matrices")
    b, (m, n) = (1 if t.dim() == 2 else t.shape[0]), t.shape[-2:]
    if m == 0 or n == 0:
        raise ValueError(f"{name} must have rows and columns")
    st = t.stride()
    if n > 1 and st[-1] != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    ld = st[-2] if m > 1 else max(n, st[-2])
    stride = st[0] if t.dim() == 3 and b > 1 else m * ld
    if ld < n or stride <= 0:
        raise ValueError(f"the rows of {name} must not overlap")
    return b, m, n, ld, stride


def orthogonalize(g, *, steps: int = 5, coefs=ORTHO_COEFS, eps: float = 1e-7, scale: float = 1.0, out=None,
                  workspace=None, stream=None):
    """scale times the orthogonalised g: X = g / (|g| + eps), then `steps` times
    X = a X + (b A + c A A) X with A = X X^T (of g's transpose where it has more
    rows than columns).

    g: (rows, cols) or (batch, rows, cols), f32 or bf16; coefs: (a, b, c), or a
    sequence of them, one for each step; out: the result to write to, which may
    be g.  workspace: a uint8 tensor to use in place of a new one
    (orthogonalize_workspace)."""
    import torch

    _tell_of_graphs(g)
    with _On(g, stream) as on:
        dt = _ar._dtype_of(g)
        b, m, n, ld, stride = _matrices(g, "g")
        flat, whole = [], True
        for c in coefs:
            one = [float(v) for v in c] if hasattr(c, "__len__") else [float(c)]
            whole = whole and len(one) == (3 if hasattr(c, "__len__") else 1)
            flat += one
        if len(flat) == 3:
            flat = flat * steps
        if not 1 <= steps <= AR_ORTHO_MAX_STEPS or len(flat) != 3 * steps or not whole:
            raise ValueError(f"steps is 1 .. {AR_ORTHO_MAX_STEPS}, with one (a, b, c) for all or one for each")
        o = torch.empty(g.shape, dtype=g.dtype, device=g.device) if out is None else out
        if o.shape != g.shape or o.dtype != g.dtype or not o.is_cuda or o.device.index != on.index:
            raise ValueError("out must be like g")
        _, _, _, ld_o, stride_o = _matrices(o, "out")
        d = ar_ortho_desc(batch=b, rows=m, cols=n, dtype=dt, steps=steps, coefs=(_F * len(flat))(*flat), eps=eps, scale=scale,
                          ld_in=ld, ld_out=ld_o, stride_in=stride, stride_out=stride_o)
        L, ws = _lib(), workspace
        if ws is None:
            ws = _workspace(L.ar_orthogonalize_workspace(ctypes.byref(d)), g)
        elif not ws.is_cuda or ws.device.index != on.index or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU of the call")
        rc = L.ar_orthogonalize(ctypes.byref(d), g.data_ptr(), o.data_ptr(), _ptr(ws),
                                0 if ws is None else ws.numel() * ws.element_size(), on.ptr)
        _ar._check(rc, "ar_orthogonalize")
    return o


def orthogonalize_workspace(batch: int, rows: int, cols: int, dtype="f32") -> int:
    """Bytes of orthogonalize's workspace."""
    d = ar_ortho_desc(batch=batch, rows=rows, cols=cols, dtype=_ar.DTYPES[dtype], steps=1, eps=0.0, scale=1.0)
    return _lib().ar_orthogonalize_workspace(ctypes.byref(d))


# ---- attention ------------------------------------------------------------------

def _heads(t, name, device, shape=None, dtype=None):
    """(tokens, heads, dim, token stride, head stride)."""
    if not t.is_cuda or t.device.index != device:
        raise ValueError(f"{name} must be on the GPU of the call")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    if t.dim() != 3 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError(f"{name} is {tuple(t.shape)}, expected {'(tokens, heads, dim)' if shape is None else shape}")
    (n, h, d), (ld, hs, one) = t.shape, t.stride()
    if h == 0 or d == 0:
        raise ValueError(f"{name} must have heads and elements")
    if d > 1 and one != 1:
        raise ValueError(f"the elements of a head of {name} must be contiguous")
    if h == 1:
        hs = d
    if n <= 1:
        ld = (h - 1) * hs + d
    if ld < d or hs < d or not (ld >= (h - 1) * hs + d or hs >= (n - 1) * ld + d):
        raise ValueError(f"the heads of {name} must not overlap")
    return n, h, d, ld, hs


def _starts(starts_q, starts_k, device):
    """(sequences, address, address)."""
    import torch

    if starts_k is None:
        starts_k = starts_q
    if starts_q is None:
        if starts_k is not None:
            raise ValueError("starts_k is given without starts_q")
        return 1, None, None
    for t, name in ((starts_q, "starts_q"), (starts_k, "starts_k")):
        if not t.is_cuda or t.device.index != device or t.dim() != 1 or not t.is_contiguous() or t.numel() < 1:
            raise ValueError(f"{name} must be a contiguous row of sequences + 1 values on the GPU of the call")
        if t.dtype != torch.int32:
            raise TypeError(f"{name} is {t.dtype}, expected torch.int32")
    if starts_q.numel() != starts_k.numel():
        raise ValueError("starts_q and starts_k must have as many sequences")
    return starts_q.numel() - 1, starts_q.data_ptr(), starts_k.data_ptr()


def _attention_desc(q, k, v, starts_q, starts_k, causal, scale, device, clear):
    n, h, dim, ld_q, hs_q = _heads(q, "q", device)
    m, hk, _, ld_k, hs_k = _heads(k, "k", device, (k.shape[0], k.shape[1], dim) if k.dim() == 3 else (0, 0, dim), q.dtype)
    _, _, _, ld_v, hs_v = _heads(v, "v", device, (m, hk, dim), q.dtype)
    if h % hk:
        raise ValueError(f"{h} heads cannot share {hk} key heads evenly")
    sequences, sq, sk = _starts(starts_q, starts_k, device)
    flags = (AR_ATTN_CAUSAL if causal else 0) | (AR_ATTN_CLEAR if clear else 0)
    d = ar_attention_desc(sequences=sequences, tokens_q=n, tokens_k=m, heads=h, kv_heads=hk, dim=dim, dtype=_ar._dtype_of(q), flags=flags,
                          scale=dim ** -0.5 if scale is None else scale, ld_q=ld_q, hs_q=hs_q, ld_k=ld_k, hs_k=hs_k, ld_v=ld_v, hs_v=hs_v)
    return d, sq, sk


def packed_attention(q, k, v, *, starts_q=None, starts_k=None, causal: bool = True, scale: Optional[float] = None, save: bool = False,
                     out=None, stream=None):
    """softmax(scale q k^T) v over packed sequences, bf16; with save also what
    packed_attention_backward needs: (o, lse).

    q: (queries, heads, dim), k and v: (keys, kv_heads, dim), dim up to 128, heads a
    multiple of kv_heads; strides are free as long as the elements of a head are
    contiguous, so all three may be parts of one tensor.  starts_q, starts_k: int32, on
    the GPU, sequences + 1 values that do not decrease: sequence i has the tokens
    starts[i] .. starts[i + 1] - 1; starts_k left out is starts_q, both left out one
    sequence.  A sequence may have no queries, as unused places between caches.
    causal: a sequence's last query sees all its keys, each one before it one less; a
    query that sees none has o = 0.  scale: 1 / sqrt(dim) unless given; above 0.
    out: o to write to; tokens of no sequence are then left as they were in it, and are
    zeros in a new one.  lse: (heads, queries) fp32, zeros there."""
    import torch

    if out is None and stream is None and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.attention(*nat.attention_fns, q, k, v, starts_q, starts_k, causal, scale, save, dev, nat.stream(dev))
        if got is not None:
            o, lse = _done(got, "ar_attention")
            return (o, lse) if save else o
    _tell_of_graphs(q, k, v)
    with _On(q, stream) as on:
        d, sq, sk = _attention_desc(q, k, v, starts_q, starts_k, causal, scale, on.index, out is None)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
        _, _, _, d.ld_o, d.hs_o = _heads(o, "out", on.index, tuple(q.shape), q.dtype)
        # zeros where the library leaves tokens of no sequence as they are
        make = torch.zeros if d.sequences == 0 or (out is not None and sq is not None) else torch.empty
        lse = make(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device) if save else None
        L = _lib()
        need = L.ar_attention_workspace_for(ctypes.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr())
        ws = _workspace(need, q)
        rc = L.ar_attention(ctypes.byref(d), q.data_ptr(), k.data_ptr(), v.data_ptr(), sq, sk, o.data_ptr(), _ptr(lse), _ptr(ws), need,
                            on.ptr)
        _ar._check(rc, "ar_attention")
        if d.sequences == 0 and out is None:
            o.zero_()
    return (o, lse) if save else o


def packed_attention_backward(do, q, k, v, o, lse, *, starts_q=None, starts_k=None, causal: bool = True, scale: Optional[float] = None,
                              need_dq: bool = True, need_dkv: bool = True, out=None, workspace=None, stream=None):
    """Gradients of packed_attention with regard to q, k and v: (dq, dk, dv); None
    for those not needed (need_dq, need_dkv).

    o, lse: from packed_attention(save=True) on the same arguments.  out: the three
    results to write to, None for new ones, which may be parts of one tensor; tokens of no
    sequence are left as they were in these, and are zeros in new ones.  workspace: a uint8
    tensor to use in place of a new one (packed_attention_backward_workspace)."""
    import torch

    _tell_of_graphs(do, q, k, v)
    with _On(q, stream) as on:
        dev = on.index
        d, sq, sk = _attention_desc(q, k, v, starts_q, starts_k, causal, scale, dev, out is None)
        _, _, _, d.ld_dout, d.hs_dout = _heads(do, "do", dev, tuple(q.shape), q.dtype)
        _, _, _, d.ld_o, d.hs_o = _heads(o, "o", dev, tuple(q.shape), q.dtype)
        if not lse.is_cuda or lse.device.index != dev or lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (d.heads, d.tokens_q):
            raise ValueError("lse must be what packed_attention(save=True) returned for these tensors")
        dq, dk, dv = (None, None, None) if out is None else out
        # zeros where the library leaves tokens of no sequence as they are
        make = torch.zeros if d.sequences == 0 or (out is not None and sq is not None) else torch.empty
        new = lambda like: make(like.shape, dtype=like.dtype, device=like.device)  # noqa: E731
        if need_dq:
            dq = new(q) if dq is None else dq
            _, _, _, d.ld_dq, d.hs_dq = _heads(dq, "dq", dev, tuple(q.shape), q.dtype)
        if need_dkv:
            dk, dv = new(k) if dk is None else dk, new(v) if dv is None else dv
            _, _, _, d.ld_dk, d.hs_dk = _heads(dk, "dk", dev, tuple(k.shape), q.dtype)
            _, _, _, d.ld_dv, d.hs_dv = _heads(dv, "dv", dev, tuple(v.shape), q.dtype)
        L, ws = _lib(), workspace
        if ws is None:
            ws = _workspace(L.ar_attention_backward_workspace(ctypes.byref(d)), q)
        elif not ws.is_cuda or ws.device.index != dev or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU of the call")
        rc = L.ar_attention_backward(
            ctypes.byref(d), do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), sq, sk,
            _ptr(dq) if need_dq else None, _ptr(dk) if need_dkv else None, _ptr(dv) if need_dkv else None, _ptr(ws),
            0 if ws is None else ws.numel() * ws.element_size(), on.ptr)
        _ar._check(rc, "ar_attention_backward")
    return dq if need_dq else None, dk if need_dkv else None, dv if need_dkv else None


def packed_attention_backward_workspace(queries: int, keys: int, heads: int, kv_heads: int, dim: int, sequences: int = 1, *,
                                        causal: Optional[bool] = None) -> int:
    """Bytes of packed_attention_backward's workspace; enough for a causal call and for one
    that is not, unless `causal` says which it is."""
    L, most = _lib(), 0
    for flags in (0, AR_ATTN_CAUSAL) if causal is None else (AR_ATTN_CAUSAL if causal else 0,):
        d = ar_attention_desc(sequences=sequences, tokens_q=queries, tokens_k=keys, heads=heads, kv_heads=kv_heads, dim=dim,
                              dtype=_ar.AR_BFLOAT16, flags=flags, scale=1.0)
        most = max(most, L.ar_attention_backward_workspace(ctypes.byref(d)))
    return most


# ---- loss over a vocabulary -------------------------------------------------------

def _target(target, tokens, device):
    """Bytes of a target."""
    import torch

    if not target.is_cuda or target.device.index != device or not target.is_contiguous() or target.numel() != tokens:
        raise ValueError(f"target must hold {tokens} contiguous values on the GPU of the call")
    if target.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"target is {target.dtype}, expected torch.int64 or torch.int32")
    return target.element_size()


def _vocab_desc(x, weight, target, first, classes, device):
    tokens, dim, ld_x = _rows(x, "x")
    if weight.dim() != 2:
        raise ValueError("weight must be a matrix")
    rows, _, ld_w = _rows(weight, "weight", dim, None, x.dtype, device)
    if rows == 0 or dim == 0:
        raise ValueError("weight must have rows and columns")
    classes = first + rows if classes is None else classes
    if first < 0 or first + rows > classes:
        raise ValueError(f"rows {first} .. {first + rows - 1} are not among {classes} classes")
    return ar_vocab_desc(tokens=tokens, dim=dim, rows=rows, first=first, classes=classes, dtype=_ar._dtype_of(x),
                         target_bytes=_target(target, tokens, device), ld_x=ld_x, ld_w=ld_w)


def _floats(t, name, shape, device):
    import torch

    if not t.is_cuda or t.device.index != device or not t.is_contiguous() or tuple(t.shape) != shape:
        raise ValueError(f"{name} must be a contiguous tensor of shape {shape} on the GPU of the call")
    if t.dtype != torch.float32:
        raise TypeError(f"{name} is {t.dtype}, expected torch.float32")
    return t


def vocab_loss(x, weight, target, *, stream=None):
    """Softmax cross entropy of each token over the classes x weight^T, without the
    logits in memory: (loss, lse), both fp32 and shaped as target; lse, the logarithm of
    the sum of the logits' exponentials, is what vocab_loss_backward needs.

    x: (..., dim), bf16; weight: (classes, dim); target: int64 or int32, one for each
    token; a target that is no class (a negative one, say) gives no loss and no gradient."""
    import torch

    if stream is None and (nat := _native()) is not None:
        dev = nat.device()
        got = nat.vocab_loss(*nat.vocab_loss_fns, x, weight, target, dev, nat.stream(dev))
        if got is not None:
            return _done(got, "ar_vocab_loss")
    _tell_of_graphs(x, weight)
    with _On(x, stream) as on:
        d = _vocab_desc(x, weight, target, 0, None, on.index)
        loss, lse = (torch.empty(target.shape, dtype=torch.float32, device=x.device) for _ in range(2))
        L = _lib()
        need = L.ar_vocab_loss_workspace(ctypes.byref(d), x.data_ptr(), weight.data_ptr())
        ws = _workspace(need, x)
        if d.tokens:
            rc = L.ar_vocab_loss(ctypes.byref(d), x.data_ptr(), weight.data_ptr(), target.data_ptr(), loss.data_ptr(), lse.data_ptr(), _ptr(ws),
                                 need, on.ptr)
            _ar._check(rc, "ar_vocab_loss")
    return loss, lse


def vocab_loss_part(x, weight, target, *, first: int, out=None, stream=None):
    """A rank's part of vocab_loss, of the classes first .. first + rows - 1 that `weight`
    has: (2, tokens) fp32, for vocab_loss_join.  out: the part to write to."""
    import torch

    _tell_of_graphs(x, weight)
    with _On(x, stream) as on:
        d = _vocab_desc(x, weight, target, first, None, on.index)  # targets behind these rows are another rank's
        part = torch.empty(2, d.tokens, dtype=torch.float32, device=x.device) if out is None else _floats(out, "out", (2, d.tokens), on.index)
        L = _lib()
        need = L.ar_vocab_loss_workspace(ctypes.byref(d), x.data_ptr(), weight.data_ptr())
        ws = _workspace(need, x)
        rc = L.ar_vocab_loss_part(ctypes.byref(d), x.data_ptr(), weight.data_ptr(), target.data_ptr(), part.data_ptr(), _ptr(ws), need, on.ptr)
        _ar._check(rc, "ar_vocab_loss_part")
    return part


def vocab_loss_join(parts, target, *, classes: int, stream=None):
    """(loss, lse) from the parts of all ranks, (ranks, 2, tokens), gathered by an
    AllReduce, say, of buffers in which each rank has filled its own."""
    import torch

    with _On(parts, stream) as on:
        if parts.dim() != 3 or parts.shape[0] < 1 or parts.shape[1] != 2:
            raise ValueError("parts must be (ranks, 2, tokens)")
        tokens = parts.shape[2]
        _floats(parts, "parts", tuple(parts.shape), on.index)
        if classes < 1:
            raise ValueError("classes must be 1 or more")
        d = ar_vocab_desc(tokens=tokens, dim=1, rows=1, first=0, classes=classes, dtype=_ar.AR_BFLOAT16,
                          target_bytes=_target(target, tokens, on.index))
        loss, lse = (torch.empty(target.shape, dtype=torch.float32, device=parts.device) for _ in range(2))
        rc = _lib().ar_vocab_loss_join(ctypes.byref(d), parts.shape[0], parts.data_ptr(), target.data_ptr(), loss.data_ptr(), lse.data_ptr(),
                                       on.ptr)
        _ar._check(rc, "ar_vocab_loss_join")
    return loss, lse


def vocab_loss_backward(dloss, x, weight, target, lse, *, first: Optional[int] = None, classes: Optional[int] = None, need_dx: bool = True,
                        need_dw: bool = True, out=None, workspace=None, stream=None):
    """Gradients of vocab_loss with regard to x and weight: (dx, dweight); None for
    those not needed (need_dx, need_dw).

    dloss: the gradient of each token's loss, fp32 and shaped as target, which may be
    expanded from one value; lse: from vocab_loss or vocab_loss_join.  first, classes: where
    `weight` is a rank's rows, as for vocab_loss_part and vocab_loss_join; dx is then that
    rank's part of the sum over the ranks.  out: the two results to write to.  workspace: a uint8 tensor to
    use in place of a new one (vocab_loss_backward_workspace)."""
    import torch

    _tell_of_graphs(dloss, x, weight)
    with _On(x, stream) as on:
        dev = on.index
        if (first is None) != (classes is None):
            raise ValueError("a rank's rows need both first and classes: targets of the other ranks' rows are told from no class by them")
        d = _vocab_desc(x, weight, target, first or 0, classes, dev)
        if not dloss.is_cuda or dloss.device.index != dev or dloss.numel() != d.tokens and dloss.numel() != 1:
            raise ValueError(f"dloss must hold {d.tokens} values, or one, on the GPU of the call")
        if dloss.dtype != torch.float32:
            raise TypeError(f"dloss is {dloss.dtype}, expected torch.float32")
        if dloss.numel() == 1 or all(s == 0 or n == 1 for n, s in zip(dloss.shape, dloss.stride())):
            stride = 0
        elif dloss.is_contiguous():
            stride = 1
        elif dloss.dim() == 1 and dloss.stride(0) > 0:
            stride = dloss.stride(0)
        else:
            raise ValueError("dloss must be a row, contiguous, or expanded from one value")
        if lse.numel() != d.tokens:
            raise ValueError(f"lse must hold {d.tokens} values")
        _floats(lse, "lse", tuple(lse.shape), dev)
        dx, dw = (None, None) if out is None else out
        if need_dx:
            dx = torch.empty_like(x, memory_format=torch.contiguous_format) if dx is None else dx
            _, _, d.ld_dx = _rows(dx, "dx", d.dim, d.tokens, x.dtype, dev)
        if need_dw:
            dw = torch.empty(d.rows, d.dim, dtype=x.dtype, device=x.device) if dw is None else dw
            _, _, d.ld_dw = _rows(dw, "dweight", d.dim, d.rows, x.dtype, dev)
        L, ws = _lib(), workspace
        if ws is None:
            ws = _workspace(L.ar_vocab_loss_backward_workspace(ctypes.byref(d), x.data_ptr(), weight.data_ptr(), need_dx, need_dw), x)
        elif not ws.is_cuda or ws.device.index != dev or not ws.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the GPU of the call")
        rc = L.ar_vocab_loss_backward(
            ctypes.byref(d), dloss.data_ptr(), stride, x.data_ptr(), weight.data_ptr(), target.data_ptr(), lse.data_ptr(),
            _ptr(dx) if need_dx else None, _ptr(dw) if need_dw else None, _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
            on.ptr)
        _ar._check(rc, "ar_vocab_loss_backward")
    return dx if need_dx else None, dw if need_dw else None


def vocab_loss_backward_workspace(x, weight, *, need_dx: bool = True, need_dw: bool = True) -> int:
    """Bytes of vocab_loss_backward's workspace for these tensors."""
    tokens, dim, ld_x = _rows(x, "x")
    rows, _, ld_w = _rows(weight, "weight", dim, None, x.dtype)
    d = ar_vocab_desc(tokens=tokens, dim=dim, rows=rows, first=0, classes=rows, dtype=_ar._dtype_of(x), target_bytes=8, ld_x=ld_x, ld_w=ld_w)
    return _lib().ar_vocab_loss_backward_workspace(ctypes.byref(d), x.data_ptr(), weight.data_ptr(), need_dx, need_dw)
