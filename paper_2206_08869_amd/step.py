"""The two ends of a training step on torch tensors: softmax cross entropy over a table of classes without its logits in memory, and updates of weights
whose gradients are made orthogonal (include/iodf.h has the formulas).

Tensors, streams, outputs and `live` are as in blocks.py. `classified` is the loss as a differentiable call; `class_loss` and
`class_loss_backward` record no graph and refuse tensors for which autograd would have to record one. `orthogonalise` and `muon_step` work on
gradients and change weights in place, as optimisers do, and have no gradient of their own.
"""
import ctypes
import functools
import math
import struct
from typing import NamedTuple

from . import binding as _b
from . import blocks as _k
from .blocks import _refuse

QUINTIC = (3.4445, -4.7750, 2.0315)  # the usual quintic step of the Muon optimiser: steep at 0, singular values end between 0.7 and 1.2

_LOSS, _ORTH, _MUON = struct.Struct("@q4iPPqq8Pqq"), struct.Struct("@5q5if3P"), struct.Struct("@3q6i6f4P")
_native = None


def _setup():
    global _native
    t = _k._torch or _k._setup()
    lib = _b.load_library()
    for block, kind in ((_LOSS, _b.ClassLossArgs), (_ORTH, _b.OrthArgs), (_MUON, _b.MuonArgs)):
        assert block.size == ctypes.sizeof(kind)
    ci, args, vp, i64 = ctypes.c_int, ctypes.c_char_p, ctypes.c_void_p, ctypes.c_int64
    for name in ("class_loss_forward", "class_loss_backward", "orthogonalise", "muon_step"):
        _k._native[name] = ctypes.CFUNCTYPE(ci, args, vp, i64, vp)(("iodf_" + name, lib))
    for name in ("orthogonalise_workspace", "muon_workspace"):
        _k._native[name] = ctypes.CFUNCTYPE(ci, args, ctypes.POINTER(i64))(("iodf_" + name, lib))
    whole = ctypes.CFUNCTYPE(ci, args, ci, ctypes.POINTER(i64))(("iodf_class_loss_workspace", lib))
    _k._native["class_loss_workspace"] = lambda block, need: whole(block, 0, need)
    _k._native["class_loss_backward_workspace"] = lambda block, need: whole(block, 1, need)
    _native = _k._native
    return t


def _run(name, workspace, block, device):
    work, need = _k._workspace(workspace, block, device)
    _k._call(name, device, block, work.data_ptr() if need else 0, need)


# ---- the loss over a table of classes ----

class ClassLoss(NamedTuple):
    """Of each row, float32: the loss, and the logarithm of the sum of its logits' exponentials, which class_loss_backward needs."""
    loss: object
    lse: object


def _loss_inputs(u, weight, target, live):
    kind, su = _k._matrix(u, "u")
    rows, cols = u.shape
    device = u.device
    if not isinstance(weight, _k._Tensor) or weight.dim() != 2 or weight.shape[0] < 1:
        _refuse("weight has to be a [classes, cols] tensor of one class or more")
    _, sw = _k._matrix(weight, "weight", (weight.shape[0], cols), u.dtype, device)
    if not isinstance(target, _k._Tensor) or target.dtype != _k._torch.int64 or tuple(target.shape) != (rows,) or target.device != device \
            or not target.is_contiguous():
        _refuse("target has to be a contiguous int64 tensor [rows] on the rows' GPU")
    return kind, su, sw, rows, cols, device, _k._live(live, rows, device)


def class_loss(u, weight, target, live=None):
    """lse = log sum_v exp(u . weight[v]) and loss = lse - u . weight[target] of each row -> ClassLoss, 0 in padded rows.

    u [rows, cols] and weight [classes, cols] have one type. No logits are kept; a target that is no class makes its row's loss NaN. In 16 bits products are exact and sums have 32
    bits. In float32 more than 64 rows are multiplied in 22 bits of each number, or down to 2^-51 of its row's or class's largest; no row sees how large the others are."""
    t = _k._torch if _native else _setup()
    kind, su, sw, rows, cols, device, lp = _loss_inputs(u, weight, target, live)
    loss, lse = t.empty(rows, dtype=_k._f32, device=device), t.empty(rows, dtype=_k._f32, device=device)
    block = _LOSS.pack(rows, weight.shape[0], cols, kind, 0, u.data_ptr(), weight.data_ptr(), su, sw, target.data_ptr(), lp, loss.data_ptr(),
                       lse.data_ptr(), 0, 0, 0, 0, cols, cols)
    _run("class_loss_forward", "class_loss_workspace", block, device)
    return ClassLoss(loss, lse)


def class_loss_backward(u, weight, target, lse, dloss, dlse=None, live=None, need=(True, True)):
    """dL/dloss and dL/dlse (float32 [rows]; either may be None) -> (dL/du, dL/dweight), in the tensors' type; lse as class_loss gave it.

    The logits are computed again, a piece of the classes at a time. need: which of the two are wanted, the others are None; a gradient's bits do not depend on it.
    What the logits' gradient is rounded to on its way goes by the tensors' type: 16 bits, in two parts where few of them make up a gradient; in float32 all of its 24 bits, as all products
    have, whatever the numbers' sizes (six products of 16 bits, so about a sixth of bfloat16's rate)."""
    t = _k._torch if _native else _setup()
    kind, su, sw, rows, cols, device, lp = _loss_inputs(u, weight, target, live)
    if lse is None:
        _refuse("lse has to be what class_loss returned")
    ep, dp, zp = _k._vector(lse, "lse", rows, device), _k._vector(dloss, "dloss", rows, device), _k._vector(dlse, "dlse", rows, device)
    du = _k._rows_like(u, su) if need[0] else None
    dw = _k._rows_like(weight, sw) if need[1] else None
    block = _LOSS.pack(rows, weight.shape[0], cols, kind, 0, u.data_ptr(), weight.data_ptr(), su, sw, target.data_ptr(), lp, 0, ep, dp, zp,
                       0 if du is None else du.data_ptr(), 0 if dw is None else dw.data_ptr(), cols, cols)
    _run("class_loss_backward", "class_loss_backward_workspace", block, device)
    return du, dw


_classified = None


def _make_classified():
    global _classified
    t = _k._torch if _native else _setup()

    class Classified(t.autograd.Function):
        @staticmethod
        def forward(ctx, u, weight, target, live):
            w = weight.to(u.dtype)
            loss, lse = class_loss(u, w, target, live)
            ctx.save_for_backward(u, w, target, live, lse)
            ctx.dtype = weight.dtype
            ctx.set_materialize_grads(False)
            return loss, lse

        @staticmethod
        @t.autograd.function.once_differentiable
        def backward(ctx, dloss, dlse):
            u, w, target, live, lse = ctx.saved_tensors
            need = ctx.needs_input_grad[:2]
            if dloss is None and dlse is None:
                return None, None, None, None
            dloss, dlse = (None if x is None else x.contiguous() for x in (dloss, dlse))
            du, dw = class_loss_backward(u, w, target, lse, dloss, dlse, live=live, need=need)
            return du, None if dw is None else dw.to(ctx.dtype), None, None

    _classified = Classified
    return Classified


def classified(u, weight, target, live=None):
    """class_loss as a differentiable call -> ClassLoss, whose loss and lse both have gradients (a penalty on lse keeps logits from drifting). What the
    backward pass keeps of a row is u and 4 bytes. weight may have another type than u (a 32-bit original of 16-bit products): it is rounded to u's, and the
    backward pass keeps that copy. As with any differentiable call, no eager graph of the same leaves may live while a backward pass is captured."""
    return ClassLoss(*(_classified or _make_classified()).apply(u, weight, target, live))


# ---- orthogonalised updates ----

@functools.lru_cache(maxsize=64)
def _coefficients(steps, coefficients):
    """The polynomials' numbers as C floats: one triple for all steps, or one for each."""
    each = coefficients if isinstance(coefficients[0], tuple) else (coefficients,) * steps
    if len(each) != steps or any(len(c) != 3 for c in each):
        _refuse("coefficients are three numbers, or three for each of the %d steps" % steps)
    return (ctypes.c_float * (3 * steps))(*(float(x) for c in each for x in c))


def _polynomials(steps, coefficients):
    if not isinstance(steps, int) or not 1 <= steps <= _b.IODF_ORTH_MOST:
        _refuse("steps is a number from 1 to %d" % _b.IODF_ORTH_MOST)
    try:
        flat = tuple(tuple(c) if isinstance(c, (tuple, list)) else float(c) for c in coefficients)
        return _coefficients(steps, flat)
    except (TypeError, IndexError):
        _refuse("coefficients are three numbers, or three for each step")


def _sheets(x, name, shape=None):
    """[count, rows, cols] or [rows, cols] -> type, count, rows, cols, batch and row strides."""
    if not isinstance(x, _k._Tensor) or x.dim() not in (2, 3):
        _refuse("%s has to be a float32, bfloat16 or float16 [rows, cols] or [count, rows, cols] tensor on the GPU" % name)
    if shape is not None and tuple(x.shape) != shape:
        _refuse("%s is %s, not %s" % (name, list(x.shape), list(shape)))
    if x.dim() == 2:
        kind, stride = _k._matrix(x, name)
        return kind, 1, x.shape[0], x.shape[1], x.shape[0] * stride, stride
    if x.shape[0] == 0:
        kind = _k._types.get(x.dtype)
        if kind is None or not x.is_cuda:
            _refuse("%s has to be a float32, bfloat16 or float16 tensor on the GPU" % name)
        return kind, 0, x.shape[1], x.shape[2], 0, x.shape[2]
    kind, stride = _k._matrix(x[0], name)
    (count, rows, cols), batch = x.shape, x.stride(0)
    if count > 1 and batch < (rows - 1) * stride + cols and (batch < cols or (count - 1) * batch + cols > stride):
        _refuse("the matrices of %s overlap" % name)  # neither one behind the other nor side by side between the rows of the first
    return kind, count, rows, cols, batch, stride


def _place(x, stride):
    """Address, rows, and bytes from row to row and of a row, of a [rows, cols] tensor."""
    size = x.element_size()
    return x.data_ptr(), x.shape[0], stride * size, x.shape[1] * size


def _meet(p, q):
    """Whether two places have memory in common, as far as that is easy to say: of different row strides wherever their ranges meet."""
    (at, rows, stride, cols), (other, _, other_stride, other_cols) = sorted((p, q))
    if other - at >= (rows - 1) * stride + cols:
        return False
    row, col = divmod(other - at, stride)
    return stride != other_stride or col < cols or (col + other_cols > stride and row + 1 < rows)


def _whole(x, count, rows, cols, batch, stride):
    """The place of several matrices: side by side they count as rows that are as wide as all of them, otherwise, if they are not the rows of one, as one row."""
    size = x.element_size()
    if count == 1 or batch < (rows - 1) * stride + cols:
        return x.data_ptr(), rows, stride * size, ((count - 1) * batch + cols) * size
    if batch == rows * stride:
        return x.data_ptr(), count * rows, stride * size, cols * size
    whole = ((count - 1) * batch + (rows - 1) * stride + cols) * size
    return x.data_ptr(), 1, whole, whole


def _apart(changed, read):
    """Refuses tensors, given by their places, of which one that is changed has memory in common with another."""
    places = sorted([(p, True) for p in changed] + [(p, False) for p in read])
    end, near = 0, False
    for (at, rows, stride, cols), _ in places:
        near = near or at < end
        end = max(end, at + (rows - 1) * stride + cols)
    if near and any((x or y) and _meet(p, q) for i, (p, x) in enumerate(places) for q, y in places[:i]):
        _refuse("a tensor is there twice, or overlaps another")


def orthogonalise(g, steps=5, coefficients=QUINTIC, eps=1e-7, dtype=None, out=None):
    """g / (its Frobenius norm + eps), `steps` times an odd polynomial of its singular values: nearly the orthogonal matrix next to it.

    g [rows, cols], or [count, rows, cols] for several of one shape. coefficients: (a, b, c) of X <- a X + b XX'X + c (XX')^2 X, or one triple for each
    step. dtype: the result's, g's if None; bfloat16 takes a third of the work of float32 and float16, with 11 bits of what is multiplied instead of 22.
    out may be g. At most 4096 matrices, whose shorter side is at most 16384 and longer one at most 65536, of 2^32 elements together (sides rounded up to
    multiples of 64); eps is above 0."""
    t = _k._torch if _native else _setup()
    kind, count, rows, cols, batch, stride = _sheets(g, "g")
    numbers = _polynomials(steps, coefficients)
    given = out is not None
    if not given:
        out = t.empty(g.shape, dtype=dtype or g.dtype, device=g.device)
        if out.dtype not in _k._types:
            _refuse("dtype is float32, bfloat16 or float16, not %s" % (dtype,))
    elif dtype not in (None, out.dtype) or out.device != g.device:
        _refuse("out has to have dtype, and be on g's GPU")
    to, _, _, _, out_batch, out_stride = _sheets(out, "out", tuple(g.shape))
    if min(rows, cols) < 1:
        _refuse("g has to have rows and columns")
    if given and count and (g.data_ptr(), kind, batch, stride) != (out.data_ptr(), to, out_batch, out_stride):
        _apart([_whole(out, count, rows, cols, out_batch, out_stride)], [_whole(g, count, rows, cols, batch, stride)])
    block = _ORTH.pack(count, batch, out_batch, stride, out_stride, rows, cols, kind, to, steps, eps, ctypes.addressof(numbers), g.data_ptr(),
                       out.data_ptr())
    _run("orthogonalise", "orthogonalise_workspace", block, g.device)
    if given:
        t.autograd.graph.increment_version(out)
    return out


def _each(x, name):
    x = list(x) if isinstance(x, (list, tuple)) else [x]
    for w in x:
        if not isinstance(w, _k._Tensor):
            _refuse("%s has to be a tensor or a list of tensors" % name)
    return x


def _alike(tensors, name, shape, device, dtype=None):
    """Type and row stride that the tensors share."""
    first = None
    for w in tensors:
        if w.requires_grad and not w.is_leaf and _k._torch.is_grad_enabled():
            _refuse("%s has to be what is learned itself, not computed from it" % name)
        got = (*_k._matrix(w, name, shape, dtype, device, recorded=False), w.dtype)
        if first is not None and got != first:
            _refuse("the tensors of %s have to be alike in type and layout" % name)
        first = got
    return first[:2]


def muon_step(weights, grads, momenta, rate, beta=0.95, nesterov=True, decay=0.0, scale=None, steps=5, coefficients=QUINTIC, eps=1e-7):
    """One step of an optimiser with orthogonalised updates, in place, for a weight [rows, cols] or a list of weights of one shape:
    m <- beta m + g, w <- (1 - rate decay) w - rate scale orthogonalise(g + beta m, or m without nesterov).

    momenta are contiguous float32 tensors, zeros before the first step. scale None: sqrt(max(1, rows / cols)). The numbers are part of a captured graph.
    The products are those of a result in the weights' type: bfloat16 weights take a third of the work of the others, with 11 bits of what is multiplied instead of 22 whatever the
    gradients' type. A list may be as long as it likes: as many weights go together as have 2^26 elements."""
    t = _k._torch if _native else _setup()
    weights, grads, momenta = _each(weights, "weights"), _each(grads, "grads"), _each(momenta, "momenta")
    if not len(weights) == len(grads) == len(momenta):
        _refuse("%d weights, %d gradients and %d momenta" % (len(weights), len(grads), len(momenta)))
    if not weights:
        return
    shape, device = tuple(weights[0].shape), weights[0].device
    tw, sw = _alike(weights, "weights", shape, device)
    tg, sg = _alike(grads, "grads", shape, device)
    _alike(momenta, "momenta", shape, device, _k._f32)
    rows, cols = shape
    if rows < 1 or not all(m.is_contiguous() for m in momenta):
        _refuse("weights have to have rows, and momenta to be contiguous")
    _apart([_place(w, sw) for w in weights] + [_place(m, cols) for m in momenta], [_place(g, sg) for g in grads])
    scale = math.sqrt(max(1.0, rows / cols)) if scale is None else scale
    numbers, most = _polynomials(steps, coefficients), _b.IODF_MUON_MOST
    for at in range(0, len(weights), most):
        w, g, m = weights[at:at + most], grads[at:at + most], momenta[at:at + most]
        lists = [(ctypes.c_void_p * len(w))(*(x.data_ptr() for x in part)) for part in (w, g, m)]
        block = _MUON.pack(len(w), sw, sg, rows, cols, tw, tg, steps, 1 if nesterov else 0, eps, rate, beta, decay, scale, 0.0,
                           ctypes.addressof(numbers), *(ctypes.addressof(x) for x in lists))
        _run("muon_step", "muon_workspace", block, device)
    t.autograd.graph.increment_version(weights + momenta)
