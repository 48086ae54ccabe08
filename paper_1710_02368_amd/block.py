"""Python binding of the block operators (include/agn_block.h).

Argument marshalling only: every function takes torch tensors on a ROCm
device, makes the output tensors (uninitialised memory of torch's allocator on
the current stream, which the kernels fill), and enqueues the work on the
current stream of the tensors' device without waiting.

The calls stand outside autograd, each gradient being a call of its own: what
they return is not connected to inputs that require gradients.

Matrices of rows are 2-D tensors of float32 or bfloat16 with adjacent columns
(stride(1) == 1); rows may be strided.  Other strides are refused, not copied.
``dropout`` arguments are (rate, seed, step) or (rate, seed, step, step_dev),
step_dev being a one-element int32 tensor on the device that is added to step
when the kernels run (so a replayed graph draws new masks).

A training step of a block of experts:

    r = block.route(logits, k)                            # choices, weights, plan
    xs = block.dispatch(x, r)                             # rows sorted by expert
    h = block.experts(xs, r.offsets, w1, b1, relu=True, dropout=drop)
    y = block.experts(h, r.offsets, w2, b2)
    f = block.combine(y, r)                               # weighted sum of a row's experts
    res, nxt, saved = block.norms(res, f, w_post, w_pre, gate=g, alpha=a)

and backwards: norms_backward, combine_backward, experts_backward (twice),
dispatch_backward, route_backward.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .agn import AGN_BF16, AGN_FP32, AGNError, load_library

__all__ = ["NormsSaved", "Route", "dropout", "norms", "norms_backward", "route", "route_chosen", "route_backward",
           "dispatch", "dispatch_backward", "combine", "combine_backward", "experts", "experts_backward", "EXPORTED"]

EXPORTED = [
    "agn_block_error", "agn_dropout", "agn_norms", "agn_norms_backward_workspace", "agn_norms_backward",
    "agn_route_workspace", "agn_route", "agn_route_backward", "agn_dispatch", "agn_combine",
    "agn_combine_backward", "agn_experts_workspace", "agn_experts", "agn_experts_backward_workspace",
    "agn_experts_backward",
]

_vp, _i32, _i64, _f32, _u32, _u64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                     ctypes.c_uint32, ctypes.c_uint64)


def _rows_fields(name):
    return [(name, _vp), (name + "_ld", _i64)]


_MASK = [("rate", _f32), ("step", _u32), ("seed", _u64), ("step_dev", _vp)]


class agn_dropout_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i32), ("dtype", _i32), *_rows_fields("x"), *_rows_fields("out"), *_MASK]


class agn_norms_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i32), ("dtype", _i32), ("eps", _f32), ("alpha", _f32), ("gate_kind", _i32),
                *_rows_fields("residual"), *_rows_fields("f"), *_rows_fields("gate"), ("w_post", _vp), ("w_pre", _vp),
                *_MASK, *_rows_fields("residual_out"), *_rows_fields("h"), ("rstd_post", _vp), ("rstd_pre", _vp)]


class agn_norms_grad_args(ctypes.Structure):
    _fields_ = [("fwd", agn_norms_args), *_rows_fields("dresidual_out"), *_rows_fields("dh"),
                *_rows_fields("dresidual"), *_rows_fields("df"), *_rows_fields("dgate"), ("dw_post", _vp),
                ("dw_pre", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class agn_route_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("experts", _i32), ("k", _i32), ("dtype", _i32), ("over_all", _i32),
                *_rows_fields("logits"), ("chosen", _vp), ("weights", _vp), ("offsets", _vp), ("source", _vp),
                ("slot", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class agn_route_grad_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("experts", _i32), ("k", _i32), ("dtype", _i32), ("over_all", _i32),
                *_rows_fields("logits"), ("chosen", _vp), ("weights", _vp), ("dweights", _vp),
                *_rows_fields("dlogits")]


class agn_tokens_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i32), ("k", _i32), ("dtype", _i32), ("slot", _vp), ("total", _vp),
                ("weights", _vp), *_rows_fields("x"), *_rows_fields("y"), *_rows_fields("dy"), ("dweights", _vp)]


class agn_experts_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("experts", _i32), ("inputs", _i32), ("outputs", _i32), ("dtype", _i32),
                ("relu", _i32), ("offsets", _vp), *_rows_fields("x"), *_rows_fields("w"), ("bias", _vp), *_MASK,
                *_rows_fields("out"), ("workspace", _vp), ("workspace_bytes", _i64)]


class agn_experts_grad_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("experts", _i32), ("inputs", _i32), ("outputs", _i32), ("dtype", _i32),
                ("relu_input", _i32), ("input_rate", _f32), ("offsets", _vp), *_rows_fields("x"),
                *_rows_fields("dy"), *_rows_fields("w"), *_rows_fields("dx"), ("dw", _vp), ("dbias", _vp),
                ("workspace", _vp), ("workspace_bytes", _i64)]


_lib = None
_fn = {}


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        for name in ("agn_dropout", "agn_norms", "agn_norms_backward", "agn_route", "agn_route_backward",
                     "agn_dispatch", "agn_combine", "agn_combine_backward", "agn_experts", "agn_experts_backward"):
            f = getattr(lib, name)
            f.restype, f.argtypes = _i32, [_vp, _vp]
        lib.agn_block_error.restype, lib.agn_block_error.argtypes = ctypes.c_char_p, []
        for name, args in (("agn_norms_backward_workspace", [_i64, _i32]),
                           ("agn_route_workspace", [_i64, _i32, _i32]),
                           ("agn_experts_workspace", [_i64, _i32, _i32, _i32, _i32]),
                           ("agn_experts_backward_workspace", [_i64, _i32, _i32, _i32, _i32])):
            f = getattr(lib, name)
            f.restype, f.argtypes = _i64, args
        for name in EXPORTED:
            _fn[name] = getattr(lib, name)
        _lib = lib
    return _lib


def _fail(code):
    raise AGNError(code, _library().agn_block_error().decode())


# The current stream's handle.  (The call that makes no Stream object takes
# 0.1 us, the public one 2.7 us: more than a third of a small operator's call.)
_stream_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_address = ctypes.addressof
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_strided = torch.empty_strided


# Outputs.  (Given the strides, torch makes a tensor in 1.0 us instead of 1.5.)
def _new(rows, cols, dtype, device):
    return _strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _new_vector(n, device, dtype=torch.float32):
    return _strided((n,), (1,), dtype=dtype, device=device)


def _call(name, args, index):
    """Enqueue on the current stream of device `index`."""
    if _lib is None:
        _library()
    if index == _device():
        code = _fn[name](_address(args), _stream_handle(index))
    else:
        with torch.cuda.device(index):
            code = _fn[name](_address(args), _stream_handle(index))
    if code:
        _fail(code)


def _workspace(name, device, *sizes):
    """(tensor or None, its pointer, its size)"""
    if _lib is None:
        _library()
    n = _fn[name](*sizes)
    if n <= 0:
        if n < 0:
            _fail(-1)
        return None, None, 0
    t = _new_vector(n, device, torch.uint8)
    return t, t.data_ptr(), n


_DTYPES = {torch.float32: AGN_FP32, torch.bfloat16: AGN_BF16}
_MOST = 0x7FFFFFFF  # the structs' 32-bit sizes (ctypes would drop what lies above)


def _size(n, name):
    if not 0 <= n <= _MOST:
        raise ValueError(f"{name} must be in [0, 2^31), not {n}")
    return n


def _matrix(t, name, rows=None, cols=None, like=None):
    """(pointer, row stride) of a matrix of rows, its shape, type and device checked."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        want = "2-D" if rows is None or cols is None else f"{rows} x {cols}"
        raise ValueError(f"{name} must be {want}, not {tuple(shape)}")
    if shape[1] > _MOST:
        raise ValueError(f"{name} must have fewer than 2^31 columns, not {shape[1]}")
    if like is not None:
        if t.dtype is not like.dtype or t.get_device() != like.get_device():
            raise ValueError(f"{name} must be {like.dtype} on {like.device}, not {t.dtype} on {t.device}")
    elif t.dtype not in _DTYPES or not t.is_cuda:
        raise ValueError(f"{name} must be float32 or bfloat16 on a ROCm device, not {t.dtype} on {t.device}")
    ld, step = t.stride()
    if step != 1 and shape[1] > 1 and t.numel():
        raise ValueError(f"{name}: columns must be adjacent in memory (stride 1, not {step})")
    return t.data_ptr(), ld


def _vector(t, name, shape, device, dtype=torch.float32):
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {device}, "
                         f"not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _mask(dropout, device):
    """The four fields of agn_mask."""
    if dropout is None:
        return 0.0, 0, 0, None
    rate, seed, step = dropout[:3]
    dev = dropout[3] if len(dropout) > 3 else None
    if dev is not None:
        dev = _vector(dev, "step_dev", (1,), device, torch.int32)
    return float(rate), int(step) & 0xFFFFFFFF, int(seed) & 0xFFFFFFFFFFFFFFFF, dev


# --------------------------------------------------------------------------
# dropout
# --------------------------------------------------------------------------

def dropout(x, rate: float, seed: int, step: int, out=None, step_dev=None):
    """mask * x; the gradient is dropout(dy) with the same rate, seed and step.
    out: written instead of a new tensor (may be x); like torch's own, it must
    not require gradients while they are recorded, and counts as modified."""
    xp, xld = _matrix(x, "x")
    dev = x.device
    rows, cols = x.shape
    dtype = x.dtype
    given = out is not None
    if not given:
        out = _new(rows, cols, dtype, dev)
        op, old = out.data_ptr(), cols
    else:
        op, old = _matrix(out, "out", rows, cols, like=x)
        if out.requires_grad and torch.is_grad_enabled():
            raise ValueError("out requires gradients, and the call is not recorded")
    a = agn_dropout_args(rows, cols, _DTYPES[dtype], xp, xld, op, old, *_mask((rate, seed, step, step_dev), dev))
    _call("agn_dropout", a, dev.index)
    if given:
        torch.autograd.graph.increment_version(out)
    return out


# --------------------------------------------------------------------------
# norms around a block
# --------------------------------------------------------------------------

class NormsSaved(NamedTuple):
    """What norms_backward needs: the statistics (2 x rows float32: of f and of
    residual', each where it is normed), and the call's residual, from which it
    computes residual' again in float32 (replace it by None where that tensor
    has been overwritten: then the stored residual' is used, rounded as it is)."""
    rstd: torch.Tensor
    residual: Optional[torch.Tensor]


def _gate(gate, rows, cols, like):
    if gate is None:
        return 0, None, 0
    if gate.dim() == 1:
        return 1, _vector(gate, "gate", (cols,), like.device), 0
    return (2, *_matrix(gate, "gate", rows, cols, like=like))


def norms(residual, f, w_post, w_pre, gate=None, alpha: float = 1.0, eps: float = 1e-6, dropout=None):
    """residual' = residual + alpha * gate * dropout(norm(f) * w_post) and
    h = norm(residual') * w_pre.  Returns (residual', h, saved).

    f None: residual' is residual (before the first block).  w_post None: f is
    added as it is.  w_pre None: no h (after the last block).  gate: None, a
    float32 vector of a value a column, or a matrix of residual's type."""
    rp, rld = _matrix(residual, "residual")
    rows, cols = residual.shape
    dev = residual.device
    res_out, h = residual, None
    fp = fld = rop = rold = hp = hld = wo = wi = None
    if f is not None:
        fp, fld = _matrix(f, "f", rows, cols, like=residual)
        res_out = _new(rows, cols, residual.dtype, dev)
        rop, rold = res_out.data_ptr(), cols
    if w_post is not None:
        wo = _vector(w_post, "w_post", (cols,), dev)
    if w_pre is not None:
        wi = _vector(w_pre, "w_pre", (cols,), dev)
        h = _new(rows, cols, residual.dtype, dev)
        hp, hld = h.data_ptr(), cols
    rstd = _new(2, rows, torch.float32, dev)
    rs = rstd.data_ptr()
    a = agn_norms_args(rows, cols, _DTYPES[residual.dtype], eps, alpha, *_swap_gate(_gate(gate, rows, cols, residual),
                       (rp, rld, fp, fld or 0)), wo, wi, *_mask(dropout, dev), rop, rold or 0, hp, hld or 0,
                       rs if wo else None, rs + 4 * rows if wi else None)
    _call("agn_norms", a, dev.index)
    return res_out, h, NormsSaved(rstd, residual)


def _swap_gate(gate, rows):
    """gate_kind, the matrices before the gate, the gate's matrix: the struct's order."""
    return (gate[0], *rows, gate[1], gate[2])


def norms_backward(dresidual_out, dh, residual_out, f, w_post, w_pre, saved, gate=None, alpha: float = 1.0,
                   eps: float = 1e-6, dropout=None):
    """Gradients (dresidual, df, dgate, dw_post, dw_pre) of norms, None for what
    the call did not have.  residual_out, saved: what norms returned (neither it
    nor the tensor in saved.residual changed since); dresidual_out (None: zero)
    and dh: the gradients of its two outputs."""
    op, old = _matrix(residual_out, "residual_out")
    rows, cols = residual_out.shape
    dev, dt = residual_out.device, residual_out.dtype
    fp = wo = wi = drp = hp = dfp = dgp = rpo = rpr = None
    fld = drld = hld = dgld = 0
    df = dgate = dw_post = dw_pre = None
    dres = _new(rows, cols, dt, dev)
    rs = _vector(saved.rstd, "saved.rstd", (2, rows), dev)
    if dresidual_out is not None:
        drp, drld = _matrix(dresidual_out, "dresidual_out", rows, cols, like=residual_out)
    if f is not None:
        fp, fld = _matrix(f, "f", rows, cols, like=residual_out)
        df = _new(rows, cols, dt, dev)
        dfp = df.data_ptr()
    if w_post is not None:
        wo = _vector(w_post, "w_post", (cols,), dev)
        rpo = rs
        dw_post = _new_vector(cols, dev)
    if w_pre is not None:
        wi = _vector(w_pre, "w_pre", (cols,), dev)
        rpr = rs + 4 * rows
        if dh is None:
            raise ValueError("dh must be given with w_pre")
        hp, hld = _matrix(dh, "dh", rows, cols, like=residual_out)
        dw_pre = _new_vector(cols, dev)
    rp = rld = None
    if saved.residual is not None:
        rp, rld = _matrix(saved.residual, "saved.residual", rows, cols, like=residual_out)
    elif f is None:
        rp, rld = op, old
    g = _gate(gate, rows, cols, residual_out)
    if g[0] == 1:
        dgate = _new_vector(cols, dev)
    elif g[0] == 2:
        dgate = _new(rows, cols, dt, dev)
    if dgate is not None:
        dgp, dgld = dgate.data_ptr(), cols
    ws, wsp, nws = _workspace("agn_norms_backward_workspace", dev, rows, cols)
    fwd = agn_norms_args(rows, cols, _DTYPES[dt], eps, alpha, *_swap_gate(g, (rp, rld or 0, fp, fld)), wo, wi,
                         *_mask(dropout, dev), op, old, None, 0, rpo, rpr)
    a = agn_norms_grad_args(fwd, drp, drld, hp, hld, dres.data_ptr(), cols, dfp, cols, dgp, dgld,
                            dw_post.data_ptr() if dw_post is not None else None,
                            dw_pre.data_ptr() if dw_pre is not None else None, wsp, nws)
    _call("agn_norms_backward", a, dev.index)
    return dres, df, dgate, dw_post, dw_pre


# --------------------------------------------------------------------------
# routing
# --------------------------------------------------------------------------

class Route(NamedTuple):
    """Where every row goes: chosen experts and weights (rows x k), the sorted
    plan (offsets: experts + 1; source, slot: rows * k).  All int32 but the
    float32 weights."""
    chosen: torch.Tensor
    weights: Optional[torch.Tensor]
    offsets: torch.Tensor
    source: torch.Tensor
    slot: torch.Tensor


def _route_outputs(rows, k, experts, dev):
    i32 = torch.int32
    return _new_vector(experts + 1, dev, i32), _new_vector(rows * k, dev, i32), _new(rows, k, i32, dev)


def route(logits, k: int, over_all: bool = False) -> Route:
    """The k largest logits of each row, their softmax weights (over the chosen,
    or over all experts), and the rows sorted by expert.  An expert of logit
    -inf is never chosen: -1 and weight 0 stand in its place."""
    lp, lld = _matrix(logits, "logits")
    rows, experts = logits.shape
    dev = logits.device
    _size(k, "k")
    ws, wsp, nws = _workspace("agn_route_workspace", dev, rows, experts, k)
    chosen = _new(rows, k, torch.int32, dev)
    weights = _new(rows, k, torch.float32, dev)
    offsets, source, slot = _route_outputs(rows, k, experts, dev)
    a = agn_route_args(rows, experts, k, _DTYPES[logits.dtype], int(over_all), lp, lld, chosen.data_ptr(),
                       weights.data_ptr(), offsets.data_ptr(), source.data_ptr(), slot.data_ptr(), wsp, nws)
    _call("agn_route", a, dev.index)
    return Route(chosen, weights, offsets, source, slot)


def route_chosen(chosen, weights, experts: int) -> Route:
    """The plan for choices made elsewhere: chosen rows x k int32 (an expert
    outside [0, experts): none), weights rows x k float32 or None."""
    if chosen.dim() != 2 or not chosen.is_cuda:
        raise ValueError(f"chosen must be rows x k on a ROCm device, not {tuple(chosen.shape)} on {chosen.device}")
    rows, k = chosen.shape
    dev = chosen.device
    _size(experts, "experts")
    cp = _vector(chosen, "chosen", (rows, k), dev, torch.int32)
    if weights is not None:
        _vector(weights, "weights", (rows, k), dev)
    ws, wsp, nws = _workspace("agn_route_workspace", dev, rows, experts, k)
    offsets, source, slot = _route_outputs(rows, k, experts, dev)
    a = agn_route_args(rows, experts, k, AGN_FP32, 0, None, 0, cp, None, offsets.data_ptr(), source.data_ptr(),
                       slot.data_ptr(), wsp, nws)
    _call("agn_route", a, dev.index)
    return Route(chosen, weights, offsets, source, slot)


def route_backward(logits, r: Route, dweights, over_all: bool = False):
    """Gradient of the logits from that of r.weights."""
    lp, lld = _matrix(logits, "logits")
    rows, experts = logits.shape
    dev = logits.device
    k = r.chosen.shape[1]
    _has_weights(r)
    dl = _new(rows, experts, logits.dtype, dev)
    a = agn_route_grad_args(rows, experts, k, _DTYPES[logits.dtype], int(over_all), lp, lld,
                            _vector(r.chosen, "chosen", (rows, k), dev, torch.int32),
                            _vector(r.weights, "weights", (rows, k), dev),
                            _vector(dweights, "dweights", (rows, k), dev), dl.data_ptr(), experts)
    _call("agn_route_backward", a, dev.index)
    return dl


# --------------------------------------------------------------------------
# rows to their experts and back
# --------------------------------------------------------------------------

def _has_weights(r):
    if r.weights is None:
        raise ValueError("the route has no weights")


def _tokens(name, r, rows, cols, x, y, like, weights, dy=None, dweights=None):
    k = r.slot.shape[1]
    dev = like.device
    sp = _vector(r.slot, "slot", (rows, k), dev, torch.int32)
    if (r.offsets.dtype != torch.int32 or r.offsets.device != dev or r.offsets.dim() != 1 or r.offsets.numel() < 2
            or not r.offsets.is_contiguous()):
        raise ValueError(f"offsets must be a contiguous int32 vector of experts + 1 on {dev}")
    wp = None
    if weights:
        _has_weights(r)
        wp = _vector(r.weights, "weights", (rows, k), dev)
    a = agn_tokens_args(rows, cols, k, _DTYPES[like.dtype], sp, r.offsets.data_ptr() + 4 * (r.offsets.numel() - 1), wp,
                        *x, *y, *(dy or (None, 0)), dweights)
    _call(name, a, dev.index)


def dispatch(x, r: Route):
    """The rows of x at their places, sorted by expert ((rows * k) x cols)."""
    x_ = _matrix(x, "x")
    rows, cols = x.shape
    y = _new(r.slot.numel(), cols, x.dtype, x.device)
    _tokens("agn_dispatch", r, rows, cols, x_, (y.data_ptr(), cols), x, False)
    return y


def _combine(y, r, weights):
    rows, k = r.slot.shape
    y_ = _matrix(y, "y", rows * k, y.shape[-1])
    out = _new(rows, y.shape[1], y.dtype, y.device)
    _tokens("agn_combine", r, rows, y.shape[1], (out.data_ptr(), y.shape[1]), y_, y, weights)
    return out


def combine(y, r: Route):
    """Each row's weighted sum of its places in y."""
    return _combine(y, r, True)


def dispatch_backward(dy, r: Route):
    """Gradient of dispatch: each row's sum of its places in dy."""
    return _combine(dy, r, False)


def combine_backward(dout, y, r: Route):
    """Gradients (dy, dweights) of combine."""
    d_ = _matrix(dout, "dout")
    rows, cols = dout.shape
    k = r.slot.shape[1]
    y_ = _matrix(y, "y", rows * k, cols, like=dout)
    dy = _new(rows * k, cols, y.dtype, y.device)
    dw = _new(rows, k, torch.float32, y.device)
    _tokens("agn_combine_backward", r, rows, cols, d_, y_, dout, True, (dy.data_ptr(), cols), dw.data_ptr())
    return dy, dw


# --------------------------------------------------------------------------
# the experts' products
# --------------------------------------------------------------------------

def _experts_weights(w, x):
    """(experts, outputs, inputs, pointer, row stride) of experts x outputs x
    inputs weights whose experts follow each other without a gap."""
    if w.dim() != 3 or w.dtype != x.dtype or w.device != x.device:
        raise ValueError(f"w must be experts x outputs x inputs, {x.dtype} on {x.device}")
    e, o, i = w.shape
    if max(e, o, i) > _MOST:
        raise ValueError(f"w: every size must be below 2^31, not {tuple(w.shape)}")
    se, ld, step = w.stride()
    if o == 1:
        ld = se if e > 1 else max(i, 1)
    if (step != 1 and i > 1) or (e > 1 and se != o * ld):
        raise ValueError(f"w: strides {w.stride()} (columns must be adjacent, experts outputs rows apart)")
    return e, o, i, w.data_ptr(), ld


def _experts_offsets(offsets, experts, dev):
    return _vector(offsets, "offsets", (experts + 1,), dev, torch.int32)


def experts(x, offsets, w, bias=None, relu: bool = False, dropout=None):
    """dropout(act(x w_e^T + bias_e)) of the sorted rows x, expert e's rows being
    offsets[e] .. offsets[e + 1]; rows of no expert are zero."""
    xp, xld = _matrix(x, "x")
    e, o, i, wp, wld = _experts_weights(w, x)
    rows = x.shape[0]
    if x.shape[1] != i:
        raise ValueError(f"x must have {i} columns, not {x.shape[1]}")
    dev = x.device
    dt = _DTYPES[x.dtype]
    out = _new(rows, o, x.dtype, dev)
    ws, wsp, nws = _workspace("agn_experts_workspace", dev, rows, e, i, o, dt)
    a = agn_experts_args(rows, e, i, o, dt, int(relu), _experts_offsets(offsets, e, dev), xp, xld, wp, wld,
                         _vector(bias, "bias", (e, o), dev) if bias is not None else None, *_mask(dropout, dev),
                         out.data_ptr(), o, wsp, nws)
    _call("agn_experts", a, dev.index)
    return out


def experts_backward(x, dy, offsets, w, relu_input: bool = False, input_rate: float = 0.0, need_dx: bool = True,
                     need_dw: bool = True):
    """Gradients (dx, dw, dbias) from dy, the gradient of x w_e^T + bias_e; dw
    and dbias in float32.  relu_input: x came out of a ReLU and a dropout of
    input_rate, and dx is the gradient before those.  need_dx, need_dw False:
    dx, dw None."""
    xp, xld = _matrix(x, "x")
    e, o, i, wp, wld = _experts_weights(w, x)
    rows = x.shape[0]
    if x.shape[1] != i:
        raise ValueError(f"x must have {i} columns, not {x.shape[1]}")
    yp, yld = _matrix(dy, "dy", rows, o, like=x)
    dev = x.device
    dt = _DTYPES[x.dtype]
    dx = _new(rows, i, x.dtype, dev) if need_dx else None
    dw = _strided((e, o, i), (o * i, i, 1), dtype=torch.float32, device=dev) if need_dw else None
    db = _new(e, o, torch.float32, dev)
    ws, wsp, nws = _workspace("agn_experts_backward_workspace", dev, rows, e, i, o, dt)
    a = agn_experts_grad_args(rows, e, i, o, dt, int(relu_input), input_rate, _experts_offsets(offsets, e, dev),
                              xp, xld, yp, yld, wp, wld, dx.data_ptr() if dx is not None else None, i,
                              dw.data_ptr() if dw is not None else None, db.data_ptr(), wsp, nws)
    _call("agn_experts_backward", a, dev.index)
    return dx, dw, db
