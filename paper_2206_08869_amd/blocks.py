"""Training operators of residual blocks on torch tensors: norms around a block fused with its gate and residual scale, the gated
activation, and the gradients of both and of linear layers out of 8-bit activation checkpoints (include/iodf.h has the formulas).

Tensors are [rows, cols] on one GPU with consecutive columns (any row stride); work goes to the current stream of their device, whose
allocator supplies outputs and scratch. Parameters (alpha, gate, norm weights) are float32. `live` (bool or uint8 [rows]) marks rows that
are not padding. `joined`, `projection` and `gated_projection` are the same operators as differentiable calls; the others record no graph, and
refuse activations and gradients for which autograd would have to record one.
"""
import ctypes
import struct
from typing import NamedTuple, Optional

from . import binding as _b

_ACTS = {"relu": _b.IODF_ACT_RELU, "silu": _b.IODF_ACT_SILU, "gelu": _b.IODF_ACT_GELU}
_torch = _types = _f32 = _Tensor = _stream_of = None
_native = {}

# The argument blocks as one pack() each, a few microseconds less a call than filling a ctypes.Structure field by field.
_JOIN, _GLU, _WGRAD = struct.Struct("@qq3if9P4q10P"), struct.Struct("@q3i7P6q6P"), struct.Struct("@q4iPq5Pq")


def _setup():
    """torch, and the library's entry points: on first use, since importing the package loads neither."""
    global _torch, _types, _f32, _Tensor, _stream_of
    import torch
    lib = _b.load_library()
    for block, kind in ((_JOIN, _b.JoinArgs), (_GLU, _b.GluArgs), (_WGRAD, _b.WgradArgs)):
        assert block.size == ctypes.sizeof(kind)
    ci, args, vp, i64 = ctypes.c_int, ctypes.c_char_p, ctypes.c_void_p, ctypes.c_int64
    for name, more in (("join_forward", ()), ("glu_forward", ()), ("glu_backward", ()), ("join_backward", (vp, i64)), ("weight_grad", (vp, i64))):
        _native[name] = ctypes.CFUNCTYPE(ci, args, *more, vp)(("iodf_" + name, lib))
    _native["pack"] = ctypes.CFUNCTYPE(ci, vp, ci, i64, i64, ci, vp, vp, vp, vp)(("iodf_pack", lib))
    _native["unpack"] = ctypes.CFUNCTYPE(ci, vp, vp, i64, ci, vp, ci, i64, vp)(("iodf_unpack", lib))
    for name in ("join_workspace", "weight_grad_workspace"):
        _native[name] = ctypes.CFUNCTYPE(ci, args, ctypes.POINTER(i64))(("iodf_" + name, lib))
    _types = {torch.float32: _b.IODF_T_F32, torch.bfloat16: _b.IODF_T_BF16, torch.float16: _b.IODF_T_F16}
    _f32, _Tensor = torch.float32, torch.Tensor
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _stream_of = raw or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch
    return torch


def _call(name, device, *args):
    """An entry point on the current stream of `device`, with that device current."""
    index = device.index
    if _torch.cuda.current_device() == index:
        rc = _native[name](*args, _stream_of(index))
    else:
        with _torch.cuda.device(device):
            rc = _native[name](*args, _stream_of(index))
    if rc:
        _b._check(rc)


def _workspace(name, block, device):
    need = ctypes.c_int64(0)
    rc = _native[name](block, need)
    if rc:
        _b._check(rc)
    return _torch.empty(need.value, dtype=_torch.uint8, device=device) if need.value else None, need.value


class Codes(NamedTuple):
    """A checkpoint: q int8 [rows, pitch], e uint8 [rows, pitch / 32], pitch the columns rounded up to a multiple of 32."""
    q: object
    e: object
    cols: int


class JoinSaved(NamedTuple):
    """What join_backward needs: the normalised stream x and block output n as codes, and the norms' factors, float32 [rows]."""
    x: Optional[Codes]
    n: Codes
    inv_pre: object
    inv_post: object


class JoinGrads(NamedTuple):
    dh: object
    df: object
    dalpha: object
    dgate: object
    dw_post: object
    dw_pre: object


class GluSaved(NamedTuple):
    a: Codes
    b: Codes


# ---- checks ----

def _refuse(what):
    raise ValueError("iodf: " + what)


def _matrix(x, name, shape=None, dtype=None, device=None, recorded=True):
    """Element type and row stride of a [rows, cols] tensor that the kernels take. `recorded`: autograd would record what is made of it."""
    if not isinstance(x, _Tensor) or x.dim() != 2 or x.dtype not in _types or not x.is_cuda:
        _refuse("%s has to be a float32, bfloat16 or float16 [rows, cols] tensor on the GPU" % name)
    if x.requires_grad and recorded and _torch.is_grad_enabled():
        _refuse("%s requires a gradient, and this call records no graph: take joined, projection or gated_projection, or torch.no_grad()" % name)
    r, c = x.shape
    if shape is not None and (r, c) != shape:
        _refuse("%s is %s, not %s" % (name, [r, c], list(shape)))
    if dtype is not None and x.dtype != dtype:
        _refuse("%s is %s, not %s" % (name, x.dtype, dtype))
    if device is not None and x.device != device:
        _refuse("%s is on %s, the rest on %s" % (name, x.device, device))
    stride, step = x.stride()
    if c < 1 or (r > 0 and c > 1 and step != 1):
        _refuse("%s has to have one column or more, consecutive in memory" % name)
    if r <= 1:
        stride = c
    elif stride < c:
        _refuse("the rows of %s overlap" % name)
    return _types[x.dtype], stride


def _vector(x, name, n, device):
    """Address of a contiguous float32 tensor of n values (0: none)."""
    if x is None:
        return 0
    if not isinstance(x, _Tensor) or x.dtype != _f32 or x.numel() != n or x.device != device or not x.is_contiguous():
        _refuse("%s has to be a contiguous float32 tensor of %d values on %s" % (name, n, device))
    return x.data_ptr()


def _live(live, rows, device):
    if live is None:
        return 0
    if not isinstance(live, _Tensor) or live.dtype not in (_torch.bool, _torch.uint8) or tuple(live.shape) != (rows,) or live.device != device \
            or not live.is_contiguous():
        _refuse("live has to be a contiguous bool or uint8 tensor [rows] on the rows' GPU")
    return live.data_ptr()


def _pitch(cols):
    return (cols + 31) // 32 * 32


def _codes(c, name, rows, cols, device):
    if not isinstance(c, Codes):
        _refuse("%s has to be Codes" % name)
    pitch = _pitch(cols)
    q, e, _ = c
    if not isinstance(q, _Tensor) or not isinstance(e, _Tensor) or c.cols != cols or q.dtype != _torch.int8 or e.dtype != _torch.uint8 or q.shape != (rows, pitch) or e.shape != (rows, pitch // 32) \
            or q.device != device or e.device != device or not q.is_contiguous() or not e.is_contiguous():
        _refuse("%s has to be the codes of %d x %d values on %s" % (name, rows, cols, device))
    return q.data_ptr(), e.data_ptr()


# A new tensor's sizes are arguments one by one: 1.3 us, as a tuple 1.6.

def _new_codes(rows, cols, device):
    pitch = _pitch(cols)
    return Codes(_torch.empty(rows, pitch, dtype=_torch.int8, device=device),
                 _torch.empty(rows, pitch // 32, dtype=_torch.uint8, device=device), cols)


def _rows_like(x, stride):
    """A new tensor of x's shape and type with its rows one after the other; `stride` as _matrix gave it."""
    return _torch.empty_like(x) if stride == x.shape[1] else _torch.empty(*x.shape, dtype=x.dtype, device=x.device)


# ---- checkpoints ----

def pack(x, live=None):
    """x -> Codes."""
    _torch or _setup()
    kind, stride = _matrix(x, "x", recorded=False)  # whole numbers have no gradient
    rows, cols = x.shape
    device = x.device
    lp = _live(live, rows, device)
    out = _new_codes(rows, cols, device)
    _call("pack", device, x.data_ptr(), kind, stride, rows, cols, lp, out.q.data_ptr(), out.e.data_ptr())
    return out


def unpack(codes, dtype=None):
    """What Codes stand for, as bfloat16 (default) or float32: exact in both."""
    t = _torch or _setup()
    dtype = t.bfloat16 if dtype is None else dtype
    if dtype not in (t.bfloat16, t.float32):
        _refuse("codes are unpacked to bfloat16 or float32")
    if not isinstance(codes, Codes) or not isinstance(codes.q, _Tensor) or codes.q.dim() != 2:
        _refuse("codes has to be Codes")
    rows, cols, device = codes.q.shape[0], codes.cols, codes.q.device
    qp, ep = _codes(codes, "codes", rows, cols, device)
    if device.type != "cuda":
        _refuse("codes have to be on the GPU")
    y = t.empty(rows, cols, dtype=dtype, device=device)
    _call("unpack", device, qp, ep, rows, cols, y.data_ptr(), _types[dtype], cols)
    return y


# ---- join ----

def _join_params(rows, cols, device, alpha, gate, w_post, w_pre, live):
    gate_rows, gp = rows, 0
    if gate is not None:
        if not isinstance(gate, _Tensor) or gate.dim() not in (1, 2):
            _refuse("gate has to be a float32 tensor [cols] or [groups, cols]")
        groups = 1 if gate.dim() == 1 else gate.shape[0]
        if gate.shape[-1] != cols or groups < 1 and rows or groups > 1 and rows % groups:
            _refuse("gate is %s: [cols] or [groups, cols] is wanted, groups that divide the %d rows" % (list(gate.shape), rows))
        gate_rows = rows // groups if groups else 0
        gp = _vector(gate, "gate", groups * cols, device)
    return (gate_rows or 1, _vector(alpha, "alpha", 1, device), gp, _vector(w_post, "w_post", cols, device), _vector(w_pre, "w_pre", cols, device),
            _live(live, rows, device))


def join(h, f, alpha=None, gate=None, w_post=None, w_pre=None, live=None, eps=1e-6, save=True, h_out=None):
    """h' = h + alpha * gate * w_post * f / rms(f) and u = w_pre * h' / rms(h') -> (h', u, JoinSaved).

    gate is [cols] or [groups, cols], rows in groups of equal length. w_post None: no norm behind the block; w_pre None: no u (None).
    save=False keeps nothing (None), for inference. h_out may be h."""
    t = _torch or _setup()
    th, sh = _matrix(h, "h")
    shape = rows, cols = tuple(h.shape)
    device = h.device
    tf, sf = _matrix(f, "f", shape, None, device)
    gate_rows, ap, gp, wop, wip, lp = _join_params(rows, cols, device, alpha, gate, w_post, w_pre, live)
    given = h_out is not None
    if not given:
        h_out, so = _rows_like(h, sh), cols
    else:
        _, so = _matrix(h_out, "h_out", shape, h.dtype, device)
    u = _rows_like(f, sf) if w_pre is not None else None
    saved, c = None, (0, 0, 0, 0, 0, 0)
    if save:
        x, n = _new_codes(rows, cols, device) if w_pre is not None else None, _new_codes(rows, cols, device)
        inv_pre = t.empty(rows, dtype=_f32, device=device) if x else None
        inv_post = t.empty(rows, dtype=_f32, device=device) if w_post is not None else None
        saved = JoinSaved(x, n, inv_pre, inv_post)
        c = (x.q.data_ptr() if x else 0, x.e.data_ptr() if x else 0, n.q.data_ptr(), n.e.data_ptr(), inv_pre.data_ptr() if x else 0,
             inv_post.data_ptr() if w_post is not None else 0)
    _call("join_forward", device, _JOIN.pack(rows, gate_rows, cols, th, tf, eps, ap, gp, wop, wip, lp, h.data_ptr(), f.data_ptr(), h_out.data_ptr(),
                                             u.data_ptr() if u is not None else 0, sh, sf, so, cols, *c, 0, 0, 0, 0))
    if given:
        t.autograd.graph.increment_version(h_out)
    return h_out, u, saved


def join_backward(saved, dh, du, alpha=None, gate=None, w_post=None, w_pre=None, live=None, block_dtype=None):
    """dL/dh' and dL/du (None where join gave no u) -> JoinGrads; df has du's type, or block_dtype."""
    t = _torch or _setup()
    th, sh = _matrix(dh, "dh")
    shape = rows, cols = tuple(dh.shape)
    device = dh.device
    if (du is None) != (w_pre is None):
        _refuse("du belongs to w_pre: both or none")
    if not isinstance(saved, JoinSaved):
        _refuse("saved has to be JoinSaved, which join returns with save=True")
    block_dtype = getattr(du, "dtype", None) if du is not None else block_dtype or dh.dtype
    if block_dtype not in _types:
        _refuse("block_dtype is float32, bfloat16 or float16, not %s" % (block_dtype,))
    tf, sf = _matrix(du, "du", shape, block_dtype, device) if du is not None else (_types[block_dtype], cols)
    gate_rows, ap, gp, wop, wip, lp = _join_params(rows, cols, device, alpha, gate, w_post, w_pre, live)
    xq, xe = _codes(saved.x, "saved.x", rows, cols, device) if w_pre is not None else (0, 0)
    nq, ne = _codes(saved.n, "saved.n", rows, cols, device)
    ipre = _vector(saved.inv_pre, "saved.inv_pre", rows, device) if w_pre is not None else 0
    ipost = _vector(saved.inv_post, "saved.inv_post", rows, device) if w_post is not None else 0
    if rows and (w_pre is not None and saved.inv_pre is None or w_post is not None and saved.inv_post is None):
        _refuse("saved lacks a norm's factors")
    dh_out = _rows_like(dh, sh)
    df = t.empty(rows, cols, dtype=block_dtype, device=device) if du is None else _rows_like(du, sf)
    fresh = t.empty_like if rows else t.zeros_like  # of no rows the kernels fill one gate's gradient, however many gates there are
    grads = [None if p is None else fresh(p) for p in (alpha, gate, w_post, w_pre)]
    block = _JOIN.pack(rows, gate_rows, cols, th, tf, 1.0, ap, gp, wop, wip, lp, dh.data_ptr(), du.data_ptr() if du is not None else 0,
                       dh_out.data_ptr(), df.data_ptr(), sh, sf, cols, cols, xq, xe, nq, ne, ipre, ipost,
                       *[0 if g is None else g.data_ptr() for g in grads])
    work, need = _workspace("join_workspace", block, device)
    _call("join_backward", device, block, work.data_ptr(), need)  # it always needs some
    return JoinGrads(dh_out, df, *grads)


# ---- gated activation ----

def _act(act):
    if act not in _ACTS:
        _refuse("act is one of %s" % ", ".join(sorted(_ACTS)))
    return _ACTS[act]


def glu(a, b, act="silu", live=None, save=True):
    """y = act(a) * b -> (y, GluSaved or None)."""
    _torch or _setup()
    kind, sa = _matrix(a, "a")
    shape = rows, cols = tuple(a.shape)
    device = a.device
    _, sb = _matrix(b, "b", shape, a.dtype, device)
    code, lp = _act(act), _live(live, rows, device)
    y = _rows_like(a, sa)
    saved, c = None, (0, 0, 0, 0)
    if save:
        saved = GluSaved(_new_codes(rows, cols, device), _new_codes(rows, cols, device))
        c = (saved.a.q.data_ptr(), saved.a.e.data_ptr(), saved.b.q.data_ptr(), saved.b.e.data_ptr())
    _call("glu_forward", device, _GLU.pack(rows, cols, kind, code, lp, a.data_ptr(), b.data_ptr(), y.data_ptr(), 0, 0, 0, sa, sb, cols, 0, 0, 0, *c, 0, 0))
    return y, saved


def _glu_backward(saved, dy, act, live, rebuild):
    """The gradients of a and b side by side, [rows, 2 cols], and the Codes of y."""
    t = _torch or _setup()
    kind, sd = _matrix(dy, "dy")
    rows, cols = dy.shape
    device = dy.device
    if not isinstance(saved, GluSaved):
        _refuse("saved has to be GluSaved, which glu returns with save=True")
    aq, ae = _codes(saved.a, "saved.a", rows, cols, device)
    bq, be = _codes(saved.b, "saved.b", rows, cols, device)
    code, lp = _act(act), _live(live, rows, device)
    dab = t.empty(rows, 2 * cols, dtype=dy.dtype, device=device)
    y = _new_codes(rows, cols, device) if rebuild else None
    da = dab.data_ptr()
    _call("glu_backward", device, _GLU.pack(rows, cols, kind, code, lp, 0, 0, 0, dy.data_ptr(), da, da + cols * dab.element_size(), 0, 0, 0, sd,
                                            2 * cols, 2 * cols, aq, ae, bq, be, y.q.data_ptr() if y else 0, y.e.data_ptr() if y else 0))
    return dab, y


def glu_backward(saved, dy, act="silu", live=None, rebuild=True):
    """dL/dy -> (dL/da, dL/db, Codes of y or None). The two gradients are the halves of one [rows, 2 cols] tensor."""
    dab, y = _glu_backward(saved, dy, act, live, rebuild)
    cols = dy.shape[1]
    return dab[:, :cols], dab[:, cols:], y


# ---- weight gradient ----

def weight_grad(codes, dy, col_scale=None, live=None, out=None, accumulate=False):
    """float32 [dy's columns, codes' columns]: (accumulate: out +) dy^T X * col_scale, X what the codes stand for."""
    t = _torch or _setup()
    kind, sd = _matrix(dy, "dy")
    rows, n_out = dy.shape
    device = dy.device
    if not isinstance(codes, Codes):
        _refuse("codes has to be Codes")
    cols = codes.cols
    qp, ep = _codes(codes, "codes", rows, cols, device)
    sp, lp = _vector(col_scale, "col_scale", cols, device), _live(live, rows, device)
    given = out is not None
    if not given:
        if accumulate:
            _refuse("accumulate adds to out: pass it")
        out, so = t.empty(n_out, cols, dtype=_f32, device=device), cols
    else:
        _, so = _matrix(out, "out", (n_out, cols), _f32, device)
    block = _WGRAD.pack(rows, cols, n_out, kind, 1 if accumulate else 0, dy.data_ptr(), sd, qp, ep, sp, lp, out.data_ptr(), so)
    work, need = _workspace("weight_grad_workspace", block, device)
    _call("weight_grad", device, block, work.data_ptr() if need else 0, need)
    if given:
        t.autograd.graph.increment_version(out)
    return out


# ---- differentiable calls ----

_functions = None


def _make_functions():
    """The autograd functions: made on first use, since importing the package does not import torch."""
    global _functions
    if _functions is not None:
        return _functions
    t = _torch or _setup()

    def rows_first(x):
        return x if x.stride(-1) == 1 and (x.shape[0] <= 1 or x.stride(0) >= x.shape[1]) else x.contiguous()

    once = t.autograd.function.once_differentiable

    # Checkpoints and the mask are kept as saved tensors, which the backward pass lets go and in which a change in place is an error.

    class Joined(t.autograd.Function):
        @staticmethod
        def forward(ctx, h, f, alpha, gate, w_post, w_pre, live, eps, hold):
            h2, u, saved = join(h, f, alpha, gate, w_post, w_pre, live=live, eps=eps, save=True)
            x, n, inv_pre, inv_post = saved
            ctx.save_for_backward(alpha, gate, w_post, w_pre, live, *(x[:2] if x else (None, None)), *n[:2], inv_pre, inv_post)
            ctx.block = f.dtype
            hold.append(saved)
            return (h2, u) if u is not None else h2

        @staticmethod
        @once
        def backward(ctx, dh, du=None):
            *params, live, xq, xe, nq, ne, inv_pre, inv_post = ctx.saved_tensors
            cols = dh.shape[1]
            saved = JoinSaved(None if xq is None else Codes(xq, xe, cols), Codes(nq, ne, cols), inv_pre, inv_post)
            g = join_backward(saved, rows_first(dh), None if du is None else rows_first(du), *params, live=live, block_dtype=ctx.block)
            return (*g, None, None, None)

    class Projection(t.autograd.Function):
        @staticmethod
        def forward(ctx, u, weight, codes, col_scale, live, learns):
            w = weight.to(u.dtype)
            if learns and not isinstance(codes, Codes):
                _refuse("codes has to be Codes")
            ctx.save_for_backward(w, col_scale, live, *(codes[:2] if learns else (None, None)))
            ctx.cols, ctx.dtype = codes.cols if learns else 0, weight.dtype
            return u @ w.t()

        @staticmethod
        @once
        def backward(ctx, dy):
            w, col_scale, live, q, e = ctx.saved_tensors
            dy, to_u, to_weight = rows_first(dy), *ctx.needs_input_grad[:2]
            dw = weight_grad(Codes(q, e, ctx.cols), dy, col_scale=col_scale, live=live).to(ctx.dtype) if to_weight else None
            return dy @ w.to(dy.dtype) if to_u else None, dw, None, None, None, None  # autocast may have given the product another type than u's

    class GatedProjection(t.autograd.Function):
        @staticmethod
        def forward(ctx, ab, weight, act, live, recorded):
            cols = ab.shape[1] // 2
            y, saved = glu(ab[:, :cols], ab[:, cols:], act, live=live, save=recorded)
            w = weight.to(y.dtype)
            if recorded:
                ctx.save_for_backward(w, live, *saved.a[:2], *saved.b[:2])
                ctx.cols, ctx.act, ctx.dtype = cols, act, weight.dtype
            return y @ w.t()

        @staticmethod
        @once
        def backward(ctx, do):
            w, live, aq, ae, bq, be = ctx.saved_tensors
            do = rows_first(do)
            saved = GluSaved(Codes(aq, ae, ctx.cols), Codes(bq, be, ctx.cols))
            to_weight = ctx.needs_input_grad[1]
            dab, y = _glu_backward(saved, do @ w.to(do.dtype), ctx.act, live, to_weight)
            return dab, weight_grad(y, do, live=live).to(ctx.dtype) if to_weight else None, None, None, None

    _functions = (Joined, Projection, GatedProjection)
    return _functions


def joined(h, f, alpha=None, gate=None, w_post=None, w_pre=None, live=None, eps=1e-6):
    """join() as a differentiable call -> (h', u, Codes of x): the codes and w_pre go to the projection that reads u. They are an answer of this
    call and made in every case: join(save=False) is the form that keeps nothing."""
    hold = []
    out = _make_functions()[0].apply(h, f, alpha, gate, w_post, w_pre, live, eps, hold)
    return (*out, hold[0].x) if w_pre is not None else (out, None, None)


def projection(u, weight, codes, col_scale=None, live=None):
    """u @ weight.T, differentiable, which keeps no u: the weight's gradient reads codes, which stand for u / col_scale."""
    call = _make_functions()[1].apply
    return call(u, weight, codes, col_scale, live, _torch.is_grad_enabled() and weight.requires_grad)


def gated_projection(ab, weight, act="silu", live=None):
    """(act(a) * b) @ weight.T for the halves a, b of ab, differentiable, which keeps a and b in 8 bits and no product."""
    call = _make_functions()[2].apply
    return call(ab, weight, act, live, _torch.is_grad_enabled() and (ab.requires_grad or weight.requires_grad))
