"""Training operators of residual blocks on torch tensors: norms around a block fused with its gate and residual scale, the gated
activation, and the gradients of both and of linear layers out of 8-bit activation checkpoints (include/iodf.h has the formulas).

Tensors are [rows, cols] on one GPU with consecutive columns (any row stride); work goes to the current stream of their device, whose
allocator supplies outputs and scratch. Parameters (alpha, gate, norm weights) are float32. `live` (bool or uint8 [rows]) marks rows that
are not padding. `joined`, `projection` and `gated_projection` are the same operators as differentiable calls.
"""
import ctypes
from typing import NamedTuple, Optional

from . import binding as _b

_ACTS = {"relu": _b.IODF_ACT_RELU, "silu": _b.IODF_ACT_SILU, "gelu": _b.IODF_ACT_GELU}
_torch, _types = None, None


def _t():
    global _torch, _types
    if _torch is None:
        import torch
        _types = {torch.float32: _b.IODF_T_F32, torch.bfloat16: _b.IODF_T_BF16, torch.float16: _b.IODF_T_F16}
        _torch = torch
    return _torch


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


def _matrix(x, name, rows=None, cols=None, dtype=None):
    """Element type and row stride of a [rows, cols] tensor that the kernels take."""
    t = _t()
    if not isinstance(x, t.Tensor) or not x.is_cuda or x.dim() != 2 or x.dtype not in _types:
        _refuse("%s has to be a float32, bfloat16 or float16 [rows, cols] tensor on the GPU" % name)
    r, c = x.shape
    if c < 1 or (r > 0 and c > 1 and x.stride(1) != 1):
        _refuse("%s has to have one column or more, consecutive in memory" % name)
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        _refuse("%s is %s, not [%s, %s]" % (name, list(x.shape), "rows" if rows is None else rows, "cols" if cols is None else cols))
    if dtype is not None and x.dtype != dtype:
        _refuse("%s is %s, not %s" % (name, x.dtype, dtype))
    stride = x.stride(0) if r > 1 else c
    if stride < c:
        _refuse("the rows of %s overlap" % name)
    return _types[x.dtype], stride


def _vector(x, name, shape, device, dtype=None):
    t = _t()
    if x is None:
        return None
    if not isinstance(x, t.Tensor) or x.dtype != (dtype or t.float32) or tuple(x.shape) != shape or x.device != device or not x.is_contiguous():
        _refuse("%s has to be a contiguous %s tensor of shape %s on %s" % (name, dtype or t.float32, list(shape), device))
    return x.data_ptr()


def _live(live, rows, device):
    t = _t()
    if live is None:
        return None
    if not isinstance(live, t.Tensor) or live.dtype not in (t.bool, t.uint8) or tuple(live.shape) != (rows,) or live.device != device \
            or not live.is_contiguous():
        _refuse("live has to be a contiguous bool or uint8 tensor [rows] on the rows' GPU")
    return live.data_ptr()


def _pitch(cols):
    return (cols + 31) // 32 * 32


def _codes(c, name, rows, cols, device):
    t = _t()
    if not isinstance(c, Codes):
        _refuse("%s has to be Codes" % name)
    pitch = _pitch(cols)
    q, e = c.q, c.e
    if c.cols != cols or q.dtype != t.int8 or e.dtype != t.uint8 or tuple(q.shape) != (rows, pitch) or tuple(e.shape) != (rows, pitch // 32) \
            or q.device != device or e.device != device or not q.is_contiguous() or not e.is_contiguous():
        _refuse("%s has to be the codes of %d x %d values on %s" % (name, rows, cols, device))
    return q.data_ptr(), e.data_ptr()


def _new_codes(rows, cols, device):
    t = _t()
    pitch = _pitch(cols)
    return Codes(t.empty((rows, pitch), dtype=t.int8, device=device), t.empty((rows, pitch // 32), dtype=t.uint8, device=device), cols)


class _On:
    """The device of a call made current, and its stream."""

    def __init__(self, device):
        cuda = _t().cuda
        self.guard = cuda.device(device) if cuda.current_device() != device.index else None
        self.device = device

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return ctypes.c_void_p(_torch.cuda.current_stream(self.device).cuda_stream)

    def __exit__(self, *a):
        if self.guard is not None:
            self.guard.__exit__(*a)


def _same_device(device, **tensors):
    for name, x in tensors.items():
        if x is not None and x.device != device:
            _refuse("%s is on %s, the rest on %s" % (name, x.device, device))


# ---- checkpoints ----

def pack(x, live=None):
    """x -> Codes."""
    kind, stride = _matrix(x, "x")
    rows, cols = x.shape
    lp = _live(live, rows, x.device)
    out = _new_codes(rows, cols, x.device)
    with _On(x.device) as st:
        _b.iodf_pack(x.data_ptr(), kind, stride, rows, cols, lp, out.q.data_ptr(), out.e.data_ptr(), st)
    return out


def unpack(codes, dtype=None):
    """What Codes stand for, as bfloat16 (default) or float32: exact in both."""
    t = _t()
    dtype = t.bfloat16 if dtype is None else dtype
    if dtype not in (t.bfloat16, t.float32):
        _refuse("codes are unpacked to bfloat16 or float32")
    if not isinstance(codes, Codes):
        _refuse("codes has to be Codes")
    rows, cols, device = codes.q.shape[0], codes.cols, codes.q.device
    qp, ep = _codes(codes, "codes", rows, cols, device)
    if device.type != "cuda":
        _refuse("codes have to be on the GPU")
    y = t.empty((rows, cols), dtype=dtype, device=device)
    with _On(device) as st:
        _b.iodf_unpack(qp, ep, rows, cols, y.data_ptr(), _types[dtype], cols, st)
    return y


# ---- join ----

def _join_params(h, alpha, gate, w_post, w_pre, live):
    rows, cols = h.shape
    device = h.device
    gate_rows = rows
    if gate is not None:
        groups = 1 if gate.dim() == 1 else gate.shape[0]
        if groups < 1 and rows or groups > 1 and rows % groups:
            _refuse("gate has %d rows, which do not divide the %d rows" % (groups, rows))
        gate_rows = rows // groups if groups else 0
        gate_shape = (cols,) if gate.dim() == 1 else (groups, cols)
    return (max(gate_rows, 1), _vector(alpha, "alpha", (1,), device), None if gate is None else _vector(gate, "gate", gate_shape, device),
            _vector(w_post, "w_post", (cols,), device), _vector(w_pre, "w_pre", (cols,), device), _live(live, rows, device))


def join(h, f, alpha=None, gate=None, w_post=None, w_pre=None, live=None, eps=1e-6, save=True, h_out=None):
    """h' = h + alpha * gate * w_post * f / rms(f) and u = w_pre * h' / rms(h') -> (h', u, JoinSaved).

    gate is [cols] or [groups, cols], rows in groups of equal length. w_post None: no norm behind the block; w_pre None: no u (None).
    save=False keeps nothing (None), for inference. h_out may be h."""
    t = _t()
    th, sh = _matrix(h, "h")
    rows, cols = h.shape
    tf, sf = _matrix(f, "f", rows, cols)
    _same_device(h.device, f=f, h_out=h_out)
    gate_rows, ap, gp, wop, wip, lp = _join_params(h, alpha, gate, w_post, w_pre, live)
    if h_out is None:
        h_out = t.empty((rows, cols), dtype=h.dtype, device=h.device)
    _, so = _matrix(h_out, "h_out", rows, cols, h.dtype)
    u = t.empty((rows, cols), dtype=f.dtype, device=h.device) if w_pre is not None else None
    saved, c = None, (None,) * 6
    if save:
        x, n = _new_codes(rows, cols, h.device) if w_pre is not None else None, _new_codes(rows, cols, h.device)
        inv = t.empty((2, rows), dtype=t.float32, device=h.device)
        saved = JoinSaved(x, n, inv[0] if w_pre is not None else None, inv[1] if w_post is not None else None)
        c = (x and x.q.data_ptr(), x and x.e.data_ptr(), n.q.data_ptr(), n.e.data_ptr(), inv.data_ptr(), inv.data_ptr() + 4 * rows)
    args = _b.JoinArgs(rows, gate_rows, cols, th, tf, eps, ap, gp, wop, wip, lp, h.data_ptr(), f.data_ptr(), h_out.data_ptr(),
                       u.data_ptr() if u is not None else None, sh, sf, so, cols, *c)
    with _On(h.device) as st:
        _b.iodf_join_forward(args, st)
    return h_out, u, saved


def join_backward(saved, dh, du, alpha=None, gate=None, w_post=None, w_pre=None, live=None, block_dtype=None):
    """dL/dh' and dL/du (None where join gave no u) -> JoinGrads; df has du's type, or block_dtype."""
    t = _t()
    th, sh = _matrix(dh, "dh")
    rows, cols = dh.shape
    device = dh.device
    if (du is None) != (w_pre is None):
        _refuse("du belongs to w_pre: both or none")
    block_dtype = du.dtype if du is not None else block_dtype or dh.dtype
    tf, sf = _matrix(du, "du", rows, cols, block_dtype) if du is not None else (_types[block_dtype], cols)
    _same_device(device, du=du)
    gate_rows, ap, gp, wop, wip, lp = _join_params(dh, alpha, gate, w_post, w_pre, live)
    xq, xe = _codes(saved.x, "saved.x", rows, cols, device) if w_pre is not None else (None, None)
    nq, ne = _codes(saved.n, "saved.n", rows, cols, device)
    ipre = _vector(saved.inv_pre, "saved.inv_pre", (rows,), device) if w_pre is not None else None
    ipost = _vector(saved.inv_post, "saved.inv_post", (rows,), device) if w_post is not None else None
    if (w_pre is not None and ipre is None and rows) or (w_post is not None and ipost is None and rows):
        _refuse("saved lacks a norm's factors")
    dh_out = t.empty((rows, cols), dtype=dh.dtype, device=device)
    df = t.empty((rows, cols), dtype=block_dtype, device=device)
    grads = [None if p is None else t.empty_like(p) for p in (alpha, gate, w_post, w_pre)]
    args = _b.JoinArgs(rows, gate_rows, cols, th, tf, 1.0, ap, gp, wop, wip, lp, dh.data_ptr(), du.data_ptr() if du is not None else None,
                       dh_out.data_ptr(), df.data_ptr(), sh, sf, cols, cols, xq, xe, nq, ne, ipre, ipost,
                       *[None if g is None else g.data_ptr() for g in grads])
    with _On(device) as st:
        need = _b.iodf_join_workspace(args)
        work = t.empty((need,), dtype=t.uint8, device=device)
        _b.iodf_join_backward(args, work.data_ptr(), need, st)
    return JoinGrads(dh_out, df, *grads)


# ---- gated activation ----

def _act(act):
    if act not in _ACTS:
        _refuse("act is one of %s" % ", ".join(sorted(_ACTS)))
    return _ACTS[act]


def glu(a, b, act="silu", live=None, save=True):
    """y = act(a) * b -> (y, GluSaved or None)."""
    t = _t()
    kind, sa = _matrix(a, "a")
    rows, cols = a.shape
    _, sb = _matrix(b, "b", rows, cols, a.dtype)
    _same_device(a.device, b=b)
    code, lp = _act(act), _live(live, rows, a.device)
    y = t.empty((rows, cols), dtype=a.dtype, device=a.device)
    saved, c = None, (None,) * 4
    if save:
        saved = GluSaved(_new_codes(rows, cols, a.device), _new_codes(rows, cols, a.device))
        c = (saved.a.q.data_ptr(), saved.a.e.data_ptr(), saved.b.q.data_ptr(), saved.b.e.data_ptr())
    args = _b.GluArgs(rows, cols, kind, code, lp, a.data_ptr(), b.data_ptr(), y.data_ptr(), None, None, None, sa, sb, cols, 0, 0, 0, *c)
    with _On(a.device) as st:
        _b.iodf_glu_forward(args, st)
    return y, saved


def glu_backward(saved, dy, act="silu", live=None, rebuild=True):
    """dL/dy -> (dL/da, dL/db, Codes of y or None). The two gradients are the halves of one [rows, 2 cols] tensor."""
    t = _t()
    kind, sd = _matrix(dy, "dy")
    rows, cols = dy.shape
    device = dy.device
    aq, ae = _codes(saved.a, "saved.a", rows, cols, device)
    bq, be = _codes(saved.b, "saved.b", rows, cols, device)
    code, lp = _act(act), _live(live, rows, device)
    dab = t.empty((rows, 2 * cols), dtype=dy.dtype, device=device)
    da, db = dab[:, :cols], dab[:, cols:]
    y = _new_codes(rows, cols, device) if rebuild else None
    args = _b.GluArgs(rows, cols, kind, code, lp, None, None, None, dy.data_ptr(), da.data_ptr(), db.data_ptr(), 0, 0, 0, sd, 2 * cols,
                      2 * cols, aq, ae, bq, be, y and y.q.data_ptr(), y and y.e.data_ptr())
    with _On(device) as st:
        _b.iodf_glu_backward(args, st)
    return da, db, y


# ---- weight gradient ----

def weight_grad(codes, dy, col_scale=None, live=None, out=None, accumulate=False):
    """float32 [dy's columns, codes' columns]: (accumulate: out +) dy^T X * col_scale, X what the codes stand for."""
    t = _t()
    kind, sd = _matrix(dy, "dy")
    rows, n_out = dy.shape
    device = dy.device
    if not isinstance(codes, Codes):
        _refuse("codes has to be Codes")
    qp, ep = _codes(codes, "codes", rows, codes.cols, device)
    cols = codes.cols
    sp, lp = _vector(col_scale, "col_scale", (cols,), device), _live(live, rows, device)
    if out is None:
        if accumulate:
            _refuse("accumulate adds to out: pass it")
        out = t.empty((n_out, cols), dtype=t.float32, device=device)
    _, so = _matrix(out, "out", n_out, cols, t.float32)
    _same_device(device, out=out)
    if n_out > 1 and out.stride(0) < cols:
        _refuse("the rows of out overlap")
    args = _b.WgradArgs(rows, cols, n_out, kind, 1 if accumulate else 0, dy.data_ptr(), sd, qp, ep, sp, lp, out.data_ptr(), so)
    with _On(device) as st:
        need = _b.iodf_weight_grad_workspace(args)
        work = t.empty((need,), dtype=t.uint8, device=device) if need else None
        _b.iodf_weight_grad(args, work.data_ptr() if need else None, need, st)
    return out


# ---- differentiable calls ----

_functions = None


def _make_functions():
    """The autograd functions: made on first use, since importing the package does not import torch."""
    global _functions
    if _functions is not None:
        return _functions
    t = _t()

    def rows_first(x):
        return x if x.stride(-1) == 1 and (x.shape[0] <= 1 or x.stride(0) >= x.shape[1]) else x.contiguous()

    class Joined(t.autograd.Function):
        @staticmethod
        def forward(ctx, h, f, alpha, gate, w_post, w_pre, live, eps, hold):
            h2, u, saved = join(h, f, alpha, gate, w_post, w_pre, live=live, eps=eps, save=True)
            ctx.params, ctx.saved, ctx.live, ctx.block = (alpha, gate, w_post, w_pre), saved, live, f.dtype
            hold.append(saved)
            return (h2, u) if u is not None else h2

        @staticmethod
        def backward(ctx, dh, du=None):
            g = join_backward(ctx.saved, rows_first(dh), None if du is None else rows_first(du), *ctx.params, live=ctx.live,
                              block_dtype=ctx.block)
            return (*g, None, None, None)

    class Projection(t.autograd.Function):
        @staticmethod
        def forward(ctx, u, weight, codes, col_scale, live):
            w = weight.to(u.dtype)
            ctx.w, ctx.codes, ctx.col_scale, ctx.live, ctx.dtype = w, codes, col_scale, live, weight.dtype
            return u @ w.t()

        @staticmethod
        def backward(ctx, dy):
            dy = rows_first(dy)
            dw = weight_grad(ctx.codes, dy, col_scale=ctx.col_scale, live=ctx.live).to(ctx.dtype)
            return dy @ ctx.w, dw, None, None, None

    class GatedProjection(t.autograd.Function):
        @staticmethod
        def forward(ctx, ab, weight, act, live):
            cols = ab.shape[1] // 2
            y, saved = glu(ab[:, :cols], ab[:, cols:], act, live=live)
            w = weight.to(y.dtype)
            ctx.w, ctx.saved, ctx.act, ctx.live, ctx.dtype = w, saved, act, live, weight.dtype
            return y @ w.t()

        @staticmethod
        def backward(ctx, do):
            do = rows_first(do)
            da, db, y = glu_backward(ctx.saved, do @ ctx.w, ctx.act, live=ctx.live)
            dw = weight_grad(y, do, live=ctx.live).to(ctx.dtype)
            return da._base, dw, None, None

    _functions = (Joined, Projection, GatedProjection)
    return _functions


def joined(h, f, alpha=None, gate=None, w_post=None, w_pre=None, live=None, eps=1e-6):
    """join() as a differentiable call -> (h', u, Codes of x): the codes and w_pre go to the projection that reads u."""
    hold = []
    out = _make_functions()[0].apply(h, f, alpha, gate, w_post, w_pre, live, eps, hold)
    return (*out, hold[0].x) if w_pre is not None else (out, None, None)


def projection(u, weight, codes, col_scale=None, live=None):
    """u @ weight.T, differentiable, which keeps no u: the weight's gradient reads codes, which stand for u / col_scale."""
    return _make_functions()[1].apply(u, weight, codes, col_scale, live)


def gated_projection(ab, weight, act="silu", live=None):
    """(act(a) * b) @ weight.T for the halves a, b of ab, differentiable, which keeps a and b in 8 bits and no product."""
    return _make_functions()[2].apply(ab, weight, act, live)
