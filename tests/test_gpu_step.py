"""The loss over a table of classes and orthogonalised updates on the GPU against their plain forms in 64 bits (step_ref.py), whose bounds come from the
arithmetic: half a step of an output's own type, half a step of what is rounded on the way, a few dozen roundings of 32-bit sums."""
import ctypes

import numpy as np
import pytest

import paper_2206_08869_amd as iodf
import step_ref as ref
from test_gpu_blocks import as_type, dev, dtype, half_unit, host, near, on_gpu, torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAMES = ["bf16", "f16", "f32"]


def some(rows, classes, cols, name, seed=0, dead=None):
    """u, w, target, live as float64 / int64 / bool, exact in the type."""
    rng = np.random.default_rng(seed + rows * 31 + classes * 7 + cols)
    w = as_type(rng.standard_normal((classes, cols)) * np.exp(0.4 * rng.standard_normal(cols)) / np.sqrt(cols), name)
    target = rng.integers(0, classes, rows)
    u = as_type(rng.standard_normal((rows, cols)) + 2.0 * w[target], name)
    live = None if dead is None else np.zeros(rows, bool) if dead == "all" else rng.random(rows) >= dead
    return u, w, target, live, rng


def spoiled(u, target, live):
    """What stands in padded rows is anything."""
    u, target = u.copy(), target.copy()
    if live is not None:
        u[~live] = np.nan
        target[~live] = -(1 << 40)
    return u, target


def long(a):
    return torch().from_numpy(np.ascontiguousarray(a, np.int64)).cuda()


def check_forward(u, w, target, live, name, du=None, dw=None):
    su, st = spoiled(u, target, live)
    du = dev(su, name) if du is None else du
    r = iodf.class_loss(du, dev(w, name) if dw is None else dw, long(st), live=on_gpu(live))
    loss, lse, s = ref.loss(u, w, target, live)
    slack = ref.logit_slack(u, w, live) + 64 * U * (1 + np.abs(lse) + np.abs(s).max(1, initial=0.0))
    near(r.lse, lse, "f32", slack, "lse")
    near(r.loss, loss, "f32", 2 * slack, "loss")
    return r


SHAPES = [(1, 1, 1), (1, 2, 7), (2, 129, 8), (3, 1000, 64), (63, 31, 65), (64, 257, 200), (65, 128, 63), (129, 127, 128), (130, 1111, 72), (300, 513, 40),
          (1, 5000, 1030), (16, 4099, 512), (17, 300, 96), (700, 2, 130)]


@pytest.mark.parametrize("rows,classes,cols", SHAPES)
@pytest.mark.parametrize("name", NAMES)
def test_class_loss(rows, classes, cols, name):
    u, w, target, live, _ = some(rows, classes, cols, name)
    check_forward(u, w, target, live, name)


@pytest.mark.parametrize("dead", [0.3, "all"])
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("rows,classes,cols", [(5, 33, 64), (200, 300, 70), (260, 65, 128)])
def test_class_loss_padding(rows, classes, cols, name, dead):
    u, w, target, live, _ = some(rows, classes, cols, name, dead=dead)
    r = check_forward(u, w, target, live, name)
    assert not host(r.loss)[~live].any() and not host(r.lse)[~live].any()


@pytest.mark.parametrize("name", NAMES)
def test_class_loss_large_and_small_logits(name):
    """Logits far from 0, far apart, and all alike."""
    u, w, target, _, rng = some(90, 400, 64, name)
    u = as_type(u * np.exp(3 * rng.standard_normal((90, 1))), name)
    u[5] = 0
    check_forward(u, w, target, None, name)


def check_backward(u, w, target, live, name, dloss, dlse, **more):
    _, lse, _ = ref.loss(u, w, target, live)
    lse32 = lse.astype(np.float32)
    su, st = spoiled(u, target, live)
    on = lambda a: None if a is None else dev(np.where(live, a, np.nan) if live is not None else a)  # noqa: E731
    got = iodf.class_loss_backward(dev(su, name), dev(w, name), long(st), on(lse32), on(dloss), on(dlse), live=on_gpu(live), **more)
    du, dw, eu, ew = ref.loss_backward(u, w, target, lse32.astype(np.float64), dloss, dlse, live, name)
    if got[0] is not None:
        near(got[0], du, name, eu, "du")
    if got[1] is not None:
        near(got[1], dw, name, ew, "dweight")
    return got


def upstream(rng, rows, kind):
    one, two = rng.standard_normal(rows).astype(np.float32).astype(np.float64) / rows, rng.standard_normal(rows).astype(np.float32).astype(np.float64) / rows
    return {"loss": (one, None), "lse": (None, two), "both": (one, two), "tiny": (one * 2.0 ** -60, None)}[kind]


@pytest.mark.parametrize("rows,classes,cols", SHAPES)
@pytest.mark.parametrize("name", NAMES)
def test_class_loss_backward(rows, classes, cols, name):
    u, w, target, live, rng = some(rows, classes, cols, name)
    check_backward(u, w, target, live, name, *upstream(rng, rows, "both"))


@pytest.mark.parametrize("kind", ["loss", "lse", "tiny"])
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dead", [None, 0.3, "all"])
def test_class_loss_backward_padding(name, kind, dead):
    u, w, target, live, rng = some(150, 270, 96, name, dead=dead)
    if kind == "tiny" and name == "f16":
        return  # gradients below what half precision holds
    check_backward(u, w, target, live, name, *upstream(rng, 150, kind))


def test_class_loss_backward_gives_what_is_asked_for():
    u, w, target, _, rng = some(40, 50, 64, "bf16")
    d = upstream(rng, 40, "loss")
    whole = check_backward(u, w, target, None, "bf16", *d)
    one = check_backward(u, w, target, None, "bf16", *d, need=(True, False))
    two = check_backward(u, w, target, None, "bf16", *d, need=(False, True))
    assert one[1] is None and two[0] is None and torch().equal(one[0], whole[0]) and torch().equal(two[1], whole[1])
    assert check_backward(u, w, target, None, "bf16", *d, need=(False, False)) == (None, None)


def test_class_loss_gradient_is_its_slope():
    """The plain form's gradient against differences, in 64 bits."""
    u, w, target, live, rng = some(6, 9, 5, "f32", dead=0.2)
    d, z = upstream(rng, 6, "both")
    total = lambda u, w: (lambda r: (d * r[0] + z * r[1]).sum())(ref.loss(u, w, target, live))  # noqa: E731
    du, dw, _, _ = ref.loss_backward(u, w, target, ref.loss(u, w, target, live)[1], d, z, live, "f32")
    for x, g, call in ((u, du, lambda v: total(v, w)), (w, dw, lambda v: total(u, v))):
        for at in np.ndindex(x.shape):
            up, down = x.copy(), x.copy()
            up[at] += 1e-5
            down[at] -= 1e-5
            assert abs((call(up) - call(down)) / 2e-5 - g[at]) < 1e-8


@pytest.mark.parametrize("name", NAMES)
def test_class_loss_strides_and_any_element(name):
    """Rows with gaps that start at any element give the bits of rows of their own."""
    t = torch()
    u, w, target, _, rng = some(70, 140, 128, name)
    d, z = (dev(x) for x in upstream(rng, 70, "both"))
    base = iodf.class_loss(dev(u, name), dev(w, name), long(target))
    grads = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), base.lse, d, z)
    for gap, first in ((0, 1), (3, 0), (8, 8), (5, 3)):
        us, ws = t.full((70 * (128 + gap) + 16,), float("nan"), dtype=dtype(name), device="cuda"), t.full((140 * (128 + gap) + 16,), float("nan"), dtype=dtype(name), device="cuda")
        uv, wv = us[first:].as_strided((70, 128), (128 + gap, 1)), ws[first:].as_strided((140, 128), (128 + gap, 1))
        uv.copy_(dev(u, name)), wv.copy_(dev(w, name))
        r = iodf.class_loss(uv, wv, long(target))
        assert t.equal(r.loss, base.loss) and t.equal(r.lse, base.lse)
        assert all(t.equal(a, b) for a, b in zip(iodf.class_loss_backward(uv, wv, long(target), r.lse, d, z), grads))


@pytest.mark.parametrize("name", NAMES)
def test_class_loss_no_rows(name):
    t = torch()
    w = t.ones((5, 9), dtype=dtype(name), device="cuda")
    u = t.empty((0, 9), dtype=dtype(name), device="cuda")
    r = iodf.class_loss(u, w, long([]))
    assert r.loss.shape == r.lse.shape == (0,)
    du, dw = iodf.class_loss_backward(u, w, long([]), r.lse, r.loss)
    assert du.shape == (0, 9) and not dw.any() and dw.shape == (5, 9)


@pytest.mark.parametrize("name", NAMES)
def test_class_loss_targets_that_are_no_class(name):
    t = torch()
    u, w, target, _, _ = some(80, 90, 64, name)
    good = iodf.class_loss(dev(u, name), dev(w, name), long(target))
    bad = target.copy()
    bad[3], bad[70] = 90, -1
    r = iodf.class_loss(dev(u, name), dev(w, name), long(bad))
    rows = np.ones(80, bool)
    rows[[3, 70]] = False
    assert np.isnan(host(r.loss)[~rows]).all() and np.array_equal(host(r.loss)[rows], host(good.loss)[rows]) and t.equal(r.lse, good.lse)
    d = t.full((80,), 0.1, device="cuda")
    du, dw = iodf.class_loss_backward(dev(u, name), dev(w, name), long(bad), r.lse, d)
    assert np.isnan(host(du)[~rows]).all() and np.isfinite(host(du)[rows]).all() and np.isnan(host(dw)).all()


@pytest.mark.parametrize("name", NAMES)
def test_class_loss_nan_stays_in_its_row(name):
    t = torch()
    u, w, target, _, _ = some(80, 90, 64, name)
    u[4, 9], u[50, 60] = np.nan, np.inf
    r = iodf.class_loss(dev(u, name), dev(w, name), long(target))
    rows = np.ones(80, bool)
    rows[[4, 50]] = False
    assert np.isfinite(host(r.loss)[rows]).all() and not np.isfinite(host(r.loss)[~rows]).any()
    du, _ = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), r.lse, t.full((80,), 0.1, device="cuda"), need=(True, False))
    assert np.isfinite(host(du)[rows]).all()


def on_card(rows, classes, cols, name, seed):
    t = torch()
    gen = t.Generator("cuda").manual_seed(seed)
    w = (t.randn((classes, cols), generator=gen, device="cuda") / cols ** 0.5).to(dtype(name))
    target = t.randint(0, classes, (rows,), generator=gen, device="cuda")
    return t.randn((rows, cols), generator=gen, device="cuda").to(dtype(name)), w, target, t.randn((rows,), generator=gen, device="cuda") / rows


@pytest.mark.parametrize("rows,classes,cols,name", [(2049, 3001, 768, "bf16"), (4096, 8192, 320, "bf16"), (1000, 20011, 136, "f16"), (600, 5003, 264, "f32"),
                                                   (131072, 4500, 16, "bf16"), (70001, 700, 24, "f32")])
def test_class_loss_of_large_tables(rows, classes, cols, name):
    """Whole tiles, slices of sums, several pieces of the classes: against 64 bits on the card, in the norm: as far as half a step of g and of the result go
    (roundings are independent: their norm is what counts)."""
    t = torch()
    u, w, target, d = on_card(rows, classes, cols, name, 3)
    r = iodf.class_loss(u, w, target)
    du, dw = iodf.class_loss_backward(u, w, target, r.lse, d)
    w64, du64, dw64 = w.double(), [], t.zeros((classes, cols), dtype=t.float64, device="cuda")
    for at in range(0, rows, 8192):
        x = u[at:at + 8192].double()
        s = x @ w64.t().contiguous()
        lse = t.logsumexp(s, 1)
        here = target[at:at + 8192]
        assert (r.lse[at:at + 8192].double() - lse).abs().max() < 2e-5
        assert (r.loss[at:at + 8192].double() - (lse - s.gather(1, here[:, None])[:, 0])).abs().max() < 4e-5
        g = t.exp(s - lse[:, None])
        g.scatter_add_(1, here[:, None], -t.ones_like(g[:, :1]))
        g *= d[at:at + 8192].double()[:, None]
        du64.append(g @ w64)
        dw64 += g.t().contiguous() @ x
    most = {"bf16": 2 * 2.0 ** -9, "f16": 2 * 2.0 ** -12, "f32": 2e-6}[name]
    small = 2.0 ** -25 if name == "f16" else 0.0  # half a step of the least numbers of half precision
    for got, want in ((du, t.cat(du64)), (dw, dw64)):
        assert (got.double() - want).norm() <= most * want.norm() + small * want.numel() ** 0.5


def test_class_loss_offsets_past_32_bits():
    """A table of more than 2^32 bytes: its last classes are read and their gradients written where they belong."""
    t = torch()
    classes, cols, rows = 1 << 19, 4160, 9
    w = t.zeros((classes, cols), dtype=t.bfloat16, device="cuda")
    u = t.ones((rows, cols), dtype=t.bfloat16, device="cuda")
    w[-1] = 1.0 / 512
    w[-2, 0] = 8.0
    target = t.tensor([classes - 1, classes - 2, 0] * 3, device="cuda")
    r = iodf.class_loss(u, w, target)
    lse = np.log((classes - 2) + np.exp(4160 / 512) + np.exp(8.0))
    want = np.array([lse - 4160 / 512, lse - 8.0, lse] * 3)
    assert np.abs(host(r.loss) - want).max() < 1e-5
    du, dw = iodf.class_loss_backward(u, w, target, r.lse, t.ones(rows, device="cuda"))
    p = np.exp(np.array([4160 / 512, 8.0, 0.0]) - lse) * rows - 3
    for row, v in ((classes - 1, p[0]), (classes - 2, p[1]), (0, p[2]), (5, p[2] + 3), (classes - 3, p[2] + 3)):
        assert (dw[row].double() - v).abs().max() <= 2 * 2.0 ** -8 * abs(v) + 1e-9
    assert du.isfinite().all()


def test_classified_gradients():
    t = torch()
    u, w, target, live, rng = some(100, 77, 72, "bf16", dead=0.2)
    su, st = spoiled(u, target, live)
    ut, wt = dev(su, "bf16").requires_grad_(), dev(w).requires_grad_()  # a 32-bit original of the table
    r = iodf.classified(ut, wt, long(st), live=on_gpu(live))
    n = int(live.sum())
    (r.loss.sum() / n + 1e-2 * (r.lse ** 2).sum() / n).backward()
    lse = host(r.lse)
    d = np.full(100, np.float64(np.float32(1.0 / n)))
    z = 2e-2 * lse / n
    du, dw, eu, ew = ref.loss_backward(u, w, target, lse, d, z, live, "bf16")
    near(ut.grad, du, "bf16", eu + 4 * U * np.abs(du), "du")
    assert wt.grad.dtype == t.float32
    near(wt.grad.bfloat16(), dw, "bf16", ew + 4 * U * np.abs(dw), "dweight")
    # only one of the two is learned; only one of the results is used; nothing is
    r = iodf.classified(ut.detach(), wt, long(st), live=on_gpu(live))
    wt.grad = None
    r.lse.sum().backward()
    _, dw, _, ew = ref.loss_backward(u, w, target, lse, None, np.ones(100), live, "bf16")
    near(wt.grad.bfloat16(), dw, "bf16", ew, "dweight of lse")
    with t.no_grad():
        assert not iodf.classified(ut, wt, long(st), live=on_gpu(live)).loss.requires_grad


def test_classified_saves_what_may_not_change():
    t = torch()
    u, w, target, _, _ = some(20, 30, 64, "bf16")
    ut, wt = dev(u, "bf16").requires_grad_(), dev(w, "bf16").requires_grad_()
    r = iodf.classified(ut, wt, long(target))
    with t.no_grad():
        ut.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        r.loss.sum().backward()


def test_calls_that_record_no_graph_refuse_what_needs_one():
    t = torch()
    u, w, target, _, _ = some(20, 30, 64, "bf16")
    ut = dev(u, "bf16").requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        iodf.class_loss(ut, dev(w, "bf16"), long(target))
    with pytest.raises(ValueError, match="requires a gradient"):
        iodf.orthogonalise(ut)
    with t.no_grad():
        iodf.class_loss(ut, dev(w, "bf16"), long(target))


# ---- orthogonalised updates ----

def gradient(rng, rows, cols, rank=None):
    k = rank or max(1, min(rows, cols) // 8)
    g = rng.standard_normal((rows, k)) * np.arange(1, k + 1) ** -0.5 @ rng.standard_normal((k, cols)) / np.sqrt(k)
    return 1e-3 * (g if rank else g + 0.5 * rng.standard_normal((rows, cols)))


def check_orth(got, g, name, steps=5, coefficients=ref.QUINTIC, eps=1e-7):
    want, off = ref.orthogonalise(g, steps, coefficients, eps, parts=name != "bf16")
    d = host(got) - want
    assert np.isfinite(d).all()
    rounding = np.linalg.norm(half_unit(name, want))
    assert np.linalg.norm(d) <= rounding + off, (np.linalg.norm(d), rounding, off)


ORTH = [(1, 1), (1, 9), (7, 1), (8, 8), (33, 64), (64, 63), (65, 130), (130, 65), (128, 128), (100, 700), (700, 100), (257, 260), (520, 300)]


@pytest.mark.parametrize("rows,cols", ORTH)
@pytest.mark.parametrize("name", NAMES)
def test_orthogonalise(rows, cols, name):
    rng = np.random.default_rng(rows * 11 + cols)
    g = as_type(gradient(rng, rows, cols), "f32")
    check_orth(iodf.orthogonalise(dev(g), dtype=dtype(name)), g, name)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("to", NAMES)
def test_orthogonalise_types(name, to):
    rng = np.random.default_rng(4)
    g = as_type(1e3 * gradient(rng, 90, 140), name)
    check_orth(iodf.orthogonalise(dev(g, name), dtype=dtype(to)), g, to)


@pytest.mark.parametrize("to", NAMES)
@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_orthogonalise_any_magnitude(to, scale):
    rng = np.random.default_rng(5)
    g = as_type(gradient(rng, 96, 70) * scale, "f32")
    check_orth(iodf.orthogonalise(dev(g), dtype=dtype(to), eps=1e-37), g, to, eps=1e-37)


@pytest.mark.parametrize("to", NAMES)
def test_orthogonalise_of_low_rank_and_uneven_columns(to):
    rng = np.random.default_rng(6)
    for g in (gradient(rng, 150, 200, rank=3), gradient(rng, 200, 120) * np.exp(2 * rng.standard_normal(120)), np.outer(np.arange(1.0, 71.0), np.ones(80))):
        g = as_type(g, "f32")
        check_orth(iodf.orthogonalise(dev(g), dtype=dtype(to)), g, to)


@pytest.mark.parametrize("to", NAMES)
def test_orthogonalise_several_and_in_place(to):
    """Matrices of a batch do not see each other: the bits of calls of their own; strided, and written over their gradients."""
    t = torch()
    rng = np.random.default_rng(7)
    g = np.stack([as_type(gradient(rng, 70, 96), to) for _ in range(5)])
    one = [iodf.orthogonalise(dev(x, to)) for x in g]
    for x, y in zip(g, one):
        check_orth(y, x, to)
    wide = t.full((5, 73, 101), float("nan"), dtype=dtype(to), device="cuda")
    view = wide[:, 1:71, 3:99]
    view.copy_(dev(g.reshape(-1, 96), to).view(5, 70, 96))
    assert t.equal(iodf.orthogonalise(view), t.stack(one))
    out = iodf.orthogonalise(view, out=view)
    assert out is view and t.equal(view, t.stack(one)) and wide.isnan().sum() == wide.numel() - view.numel()


@pytest.mark.parametrize("steps,coefficients", [(1, ref.QUINTIC), (3, (1.5, -0.5, 0.0)), (8, (1.875, -1.25, 0.375)), (2, ((3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0))),
                                                (1, (0.0, 0.0, 0.0)), (1, (-2.0, 0.0, 0.0))])
@pytest.mark.parametrize("to", ["bf16", "f32"])
def test_orthogonalise_polynomials(steps, coefficients, to):
    rng = np.random.default_rng(8)
    g = as_type(gradient(rng, 80, 100), "f32")
    check_orth(iodf.orthogonalise(dev(g), steps=steps, coefficients=coefficients, dtype=dtype(to)), g, to, steps, coefficients)


def test_orthogonalise_zeros_and_nan():
    t = torch()
    g = t.zeros((3, 70, 90), device="cuda")
    g[1] = t.randn((70, 90), generator=t.Generator("cuda").manual_seed(1), device="cuda")
    g[2] = g[1]
    g[2, 5, 5] = float("nan")
    for to in NAMES:
        r = iodf.orthogonalise(g, dtype=dtype(to))
        assert not r[0].any() and r[1].isfinite().all() and r[2].isnan().all()
    assert iodf.orthogonalise(g[:0]).shape == (0, 70, 90)


@pytest.mark.parametrize("rows,cols,name", [(2048, 512, "bf16"), (512, 2048, "f32"), (1111, 1500, "bf16"), (1800, 1800, "bf16")])
def test_orthogonalise_large(rows, cols, name):
    """Larger tiles, against 64 bits on the card. What roundings of h beside the diagonal come to was taken from a simulation of them in 64 bits: 2 to 3 h."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(2)
    g = t.randn((rows, cols), generator=gen, device="cuda") * t.exp(0.4 * t.randn((cols,), generator=gen, device="cuda"))
    x = g.double() / g.double().norm()
    x = x.t().contiguous() if rows > cols else x
    for _ in range(5):
        m = x @ x.t().contiguous()
        x = 3.4445 * x + (-4.7750 * m + 2.0315 * m @ m) @ x
    x = x.t() if rows > cols else x
    r = iodf.orthogonalise(g, dtype=dtype(name))
    assert (r.double() - x).norm() <= {"bf16": 2.0 ** -9 + 4 * 2.0 ** -12, "f32": 4e-6}[name] * x.norm()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("grad", NAMES)
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(name, grad, nesterov):
    rng = np.random.default_rng(9)
    rows, cols, rate, beta, decay, scale = 90, 130, 0.05, 0.9, 0.2, 0.7
    w = [as_type(rng.standard_normal((rows, cols)) / np.sqrt(cols), name) for _ in range(3)]
    g = [as_type(gradient(rng, rows, cols), grad) for _ in range(3)]
    m = [as_type(gradient(rng, rows, cols), "f32") for _ in range(3)]
    wt, gt, mt = [dev(x, name) for x in w], [dev(x, grad) for x in g], [dev(x) for x in m]
    before = [x.clone() for x in gt]
    assert iodf.muon_step(wt, gt, mt, rate, beta=beta, nesterov=nesterov, decay=decay, scale=scale) is None
    for k in range(3):
        assert torch().equal(gt[k], before[k])
        new = np.float64(np.float32(beta)) * m[k] + g[k]
        near(mt[k], new, "f32", 2 * U * (np.abs(m[k]) + np.abs(g[k])), "momentum")
        step, off = ref.orthogonalise(g[k] + beta * new if nesterov else new, parts=name != "bf16")
        want = (1 - rate * decay) * w[k] - rate * scale * step
        d = host(wt[k]) - want
        assert np.linalg.norm(d) <= np.linalg.norm(half_unit(name, want)) + rate * scale * off + 4 * U * np.linalg.norm(w[k])


def test_muon_step_one_tensor_and_more_than_a_launch_takes():
    """A list longer than one launch takes gives each weight the bits of a call of its own."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(3)
    w = [t.randn((9, 20), generator=gen, device="cuda") for _ in range(130)]
    g = [t.randn((9, 20), generator=gen, device="cuda") for _ in range(130)]
    m = [t.zeros((9, 20), device="cuda") for _ in range(130)]
    one = [x.clone() for x in w]
    iodf.muon_step(w, g, m, 0.1)
    for k in (0, 63, 64, 129):
        own = t.zeros((9, 20), device="cuda")
        version = one[k]._version
        iodf.muon_step(one[k], g[k], own, 0.1)
        assert t.equal(one[k], w[k]) and t.equal(own, m[k]) and t.equal(own, g[k]) and one[k]._version > version
    iodf.muon_step([], [], [], 0.1)


def test_muon_step_of_parameters():
    t = torch()
    w = t.ones((16, 24), device="cuda").requires_grad_()
    g, m = t.ones((16, 24), device="cuda"), t.zeros((16, 24), device="cuda")
    iodf.muon_step(w, g, m, 0.1, scale=1.0)
    assert w.requires_grad and (w != 1).all()
    with pytest.raises(ValueError, match="learned itself"):
        iodf.muon_step(w * 2, g, m, 0.1)
    with pytest.raises(ValueError, match="twice"):
        iodf.muon_step([w, w], [g, g], [m, m.clone()], 0.1)


# ---- streams, graphs, repeated calls ----

def test_step_calls_in_a_graph_and_on_another_stream():
    """Two captured graphs of loss, gradient and update replayed in turn with eager calls between: the bits of eager calls every time."""
    t = torch()
    sets = [on_card(300, 500, 96, "bf16", s) for s in (5, 6)]
    m0 = t.zeros((500, 96), device="cuda")

    def once(u, w, target, d):
        r = iodf.class_loss(u, w, target)
        du, dw = iodf.class_loss_backward(u, w, target, r.lse, d)
        w2, m2 = w.clone(), m0.clone()
        iodf.muon_step(w2, dw, m2, 0.1)
        return r.loss, r.lse, du, dw, w2, m2

    want = [once(*s) for s in sets]
    side, graphs, outs = t.cuda.Stream(), [], []
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        again = once(*sets[0])
    t.cuda.current_stream().wait_stream(side)
    assert all(t.equal(a, b) for a, b in zip(again, want[0]))
    for s in sets:
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            outs.append(once(*s))
        graphs.append(graph)
    for turn in range(4):
        for k in (0, 1) if turn % 2 else (1, 0):
            for o in outs[k]:
                o.fill_(0)
            graphs[k].replay()
            eager = once(*sets[1 - k])
            t.cuda.synchronize()
            assert all(t.equal(a, b) for a, b in zip(outs[k], want[k])) and all(t.equal(a, b) for a, b in zip(eager, want[1 - k]))


@pytest.mark.parametrize("name", NAMES)
def test_plain_entries_give_the_bits_of_the_torch_calls(name):
    t = torch()
    u, w, target, d = on_card(50, 70, 64, name, 7)
    r = iodf.class_loss(u, w, target)
    du, dw = iodf.class_loss_backward(u, w, target, r.lse, d)
    kind = {"f32": iodf.IODF_T_F32, "bf16": iodf.IODF_T_BF16, "f16": iodf.IODF_T_F16}[name]
    st = ctypes.c_void_p(t.cuda.current_stream().cuda_stream)
    loss, lse, du2, dw2 = t.empty_like(r.loss), t.empty_like(r.lse), t.empty_like(du), t.empty_like(dw)
    a = iodf.ClassLossArgs(rows=50, classes=70, cols=64, type=kind, u=u.data_ptr(), w=w.data_ptr(), u_stride=64, w_stride=64, target=target.data_ptr(),
                           loss=loss.data_ptr(), lse=lse.data_ptr(), dloss=d.data_ptr(), du=du2.data_ptr(), dw=dw2.data_ptr(), du_stride=64, dw_stride=64)
    for backward, call in ((0, iodf.iodf_class_loss_forward), (1, iodf.iodf_class_loss_backward)):
        need = iodf.iodf_class_loss_workspace(a, backward)
        work = t.empty(max(need, 1), dtype=t.uint8, device="cuda")
        call(a, work.data_ptr(), need, st)
    assert all(t.equal(x, y) for x, y in ((loss, r.loss), (lse, r.lse), (du, du2), (dw, dw2)))
    numbers = (ctypes.c_float * 15)(*ref.QUINTIC * 5)
    want, out = iodf.orthogonalise(u), t.empty_like(u)
    o = iodf.OrthArgs(count=1, in_stride=64, out_stride=64, rows=50, cols=64, in_type=kind, out_type=kind, steps=5, eps=1e-7,
                      coefficients=ctypes.addressof(numbers), in_=u.data_ptr(), out=out.data_ptr())
    need = iodf.iodf_orthogonalise_workspace(o)
    work = t.empty(need, dtype=t.uint8, device="cuda")
    iodf.iodf_orthogonalise(o, work.data_ptr(), need, st)
    assert t.equal(out, want)
    w1, m1, w2, m2 = w.clone(), t.zeros((70, 64), device="cuda"), w.clone(), t.zeros((70, 64), device="cuda")
    iodf.muon_step(w1, dw, m1, 0.1, beta=0.9, decay=0.01, scale=0.5)
    lists = [(ctypes.c_void_p * 1)(x.data_ptr()) for x in (w2, dw, m2)]
    a = iodf.MuonArgs(count=1, weight_stride=64, grad_stride=64, rows=70, cols=64, weight_type=kind, grad_type=kind, steps=5, nesterov=1, eps=1e-7, rate=0.1,
                      beta=0.9, decay=0.01, scale=0.5, coefficients=ctypes.addressof(numbers), weights=ctypes.addressof(lists[0]),
                      grads=ctypes.addressof(lists[1]), momenta=ctypes.addressof(lists[2]))
    need = iodf.iodf_muon_workspace(a)
    work = t.empty(need, dtype=t.uint8, device="cuda")
    iodf.iodf_muon_step(a, work.data_ptr(), need, st)
    assert t.equal(w1, w2) and t.equal(m1, m2)


@pytest.mark.parametrize("count,rows,cols,name", [(8, 1344, 1400, "bf16"), (1, 700, 8200, "bf16"), (3, 1500, 1344, "f32"), (1, 4100, 4096, "bf16")])
def test_orthogonalise_every_kind_of_tile(count, rows, cols, name):
    """Shapes whose square products are cut into tiles of 192 and 256 and into pieces of tiles, against 64 bits on the card."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(4)
    g = t.randn((count, rows, cols), generator=gen, device="cuda") * t.exp(0.4 * t.randn((cols,), generator=gen, device="cuda"))
    r = iodf.orthogonalise(g, dtype=dtype(name))
    for k in {0, count - 1}:
        x = g[k].double() / g[k].double().norm()
        x = x.t().contiguous() if rows > cols else x
        for _ in range(5):
            m = x @ x.t().contiguous()
            x = 3.4445 * x + (-4.7750 * m + 2.0315 * m @ m) @ x
        x = x.t() if rows > cols else x
        assert (r[k].double() - x).norm() <= {"bf16": 2.0 ** -9 + 4 * 2.0 ** -12, "f32": 4e-6}[name] * x.norm()


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("rows,classes,cols", [(40, 300, 96), (900, 40, 130)])
def test_class_loss_gradients_of_scaled_losses(name, rows, classes, cols):
    """2^16 times dloss: 2^16 times the gradients, to the bit (of bf16, and of f16 what fits it), also where products of g exceed half precision's range."""
    t = torch()
    u, w, target, d = on_card(rows, classes, cols, name, 8)
    lse = iodf.class_loss(u, w, target).lse
    d = d * (1.0 if name == "bf16" else 2.0 ** -16)
    for less, more in zip(iodf.class_loss_backward(u, w, target, lse, d * 3), iodf.class_loss_backward(u, w, target, lse, d * 3 * 65536)):
        if name == "bf16":
            assert t.equal(less.float() * 65536, more.float())
        else:  # less has numbers below the normal range
            assert ((less.float() * 65536 - more.float()).abs() <= 2.0 ** -25 * 65536 + more.float().abs() * 2.0 ** -11).all()


@pytest.mark.parametrize("to", NAMES)
def test_orthogonalise_side_by_side(to):
    """[rows, count, cols] turned to [count, rows, cols], from and to."""
    t = torch()
    rng = np.random.default_rng(17)
    g = dev(as_type(gradient(rng, 50 * 3, 70), to), to).view(50, 3, 70)
    want = iodf.orthogonalise(g.transpose(0, 1).contiguous())
    assert t.equal(iodf.orthogonalise(g.transpose(0, 1)), want)
    out = t.full((50, 4, 70), float("nan"), dtype=g.dtype, device="cuda")
    iodf.orthogonalise(g.transpose(0, 1), out=out[:, :3].transpose(0, 1))
    assert t.equal(out[:, :3].transpose(0, 1), want) and out[:, 3].isnan().all()
    iodf.orthogonalise(g.transpose(0, 1), out=g.transpose(0, 1))
    assert t.equal(g.transpose(0, 1), want)


def test_tensors_that_overlap_are_refused():
    t = torch()
    x = t.randn((3, 60, 80), device="cuda")
    before = x.clone()
    flat = x.view(-1)
    for g, out in ((x[0, :40], x[0, 20:]), (x[:2], x[1:]), (x[0, :, :50], x[0, :, 30:]), (x[0, :59], flat[1:4721].view(59, 80)),
                   (x[0, :30], x[0].view(t.bfloat16)[:30, :80]), (x[:, :, :50], x[:, :, 30:])):
        with pytest.raises(ValueError, match="overlap"):
            iodf.orthogonalise(g, out=out)
    assert t.equal(x, before)
    m = [t.zeros((20, 80), device="cuda") for _ in range(2)]
    g = [t.randn((20, 80), device="cuda") for _ in range(2)]
    for w, grads, momenta in (([x[0, :20], x[0, 10:30]], g, m), ([x[0, :20], x[0, 20:40]], [x[0, 5:25], g[1]], m), ([x[0, :20], x[0, 20:40]], g, [m[0], m[0]]),
                              ([x[0, :20]], [x[0, :20]], m[:1])):
        with pytest.raises(ValueError, match="overlap"):
            iodf.muon_step(w, grads, momenta, 0.1)
    assert t.equal(x, before) and not any(k.any() for k in m)
    # side by side, one gradient for both, and neighbours are fine: the bits of tensors of their own
    halves, own = [x[0, :20, :40], x[0, :20, 40:]], [x[0, :20, :40].clone(), x[0, :20, 40:].clone()]
    d, m1, m2 = g[0][:, :40], [t.zeros((20, 40), device="cuda") for _ in range(2)], [t.zeros((20, 40), device="cuda") for _ in range(2)]
    iodf.muon_step(halves, [d, d], m1, 0.1)
    for k in range(2):
        iodf.muon_step(own[k], d.contiguous(), m2[k], 0.1)
        assert t.equal(halves[k], own[k]) and t.equal(m1[k], m2[k])
    y = t.randn((2, 30, 40), device="cuda")
    want = iodf.orthogonalise(y[0])
    assert t.equal(iodf.orthogonalise(y[0], out=y[1]), want)


def test_classified_captured_with_its_backward_pass():
    """Loss, gradients and the step of a weight as a captured graph, the leaves used in it alone; eager runs on copies between the replays."""
    t = torch()
    u0, w0, target, _ = on_card(200, 90, 64, "bf16", 9)
    expanded = t.full((1,), 1.0 / 200, device="cuda").expand(200)

    def once(u, w, m):
        u, w = u.detach().requires_grad_(), w.detach().requires_grad_()
        r = iodf.classified(u, w, target)
        du, dw = t.autograd.grad([r.loss, r.lse], [u, w], [expanded, 0.01 * expanded])
        with t.no_grad():
            new = w.detach().clone()
            iodf.muon_step(new, dw, m, 0.1)
        return r.loss.detach(), du, dw, new

    want = once(u0, w0, t.zeros((90, 64), device="cuda"))
    m = t.zeros((90, 64), device="cuda")
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        once(u0, w0, m)
    t.cuda.current_stream().wait_stream(side)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        got = once(u0, w0, m)
    for _ in range(3):
        m.zero_()
        for x in got:
            x.fill_(0)
        graph.replay()
        eager = once(u0, w0, t.zeros((90, 64), device="cuda"))
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(got, want)) and all(t.equal(a, b) for a, b in zip(eager, want))


def test_two_streams_at_once():
    """The same calls on two streams at a time, with workspaces of their own: the bits of calls one after the other."""
    t = torch()
    sets = [on_card(500, 700, 256, "bf16", s) for s in (11, 12)]
    g = [t.randn((300, 260), device="cuda") for _ in sets]

    def once(k):
        u, w, target, d = sets[k]
        r = iodf.class_loss(u, w, target)
        return (*r, *iodf.class_loss_backward(u, w, target, r.lse, d), iodf.orthogonalise(g[k]))

    want = [once(k) for k in range(2)]
    t.cuda.synchronize()
    streams, got = [t.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(10):
        for k, s in enumerate(streams):
            with t.cuda.stream(s):
                got[k].append(once(k))
    t.cuda.synchronize()
    assert all(t.equal(a, b) for k in range(2) for run in got[k] for a, b in zip(run, want[k]))


@pytest.mark.parametrize("rows,classes,cols", [(3, 79, 8064), (2, 1031, 7360), (60, 200, 4100), (150, 140, 2050)])
@pytest.mark.parametrize("name", NAMES)
def test_class_loss_of_few_logits_and_long_rows(rows, classes, cols, name):
    """The columns are split among workgroups: forward, gradients, padding."""
    u, w, target, live, rng = some(rows, classes, cols, name, seed=3, dead=0.2)
    check_forward(u, w, target, live, name)
    check_backward(u, w, target, live, name, *upstream(rng, rows, "both"))


@pytest.mark.parametrize("rows,cols", [(65, 65), (128, 128), (128, 65), (70, 127), (100, 101)])
@pytest.mark.parametrize("to", NAMES)
def test_orthogonalise_one_block(rows, cols, to):
    """Matrices that fit a workgroup's LDS: several, tall and wide, strided and in place; the step of an optimiser the same."""
    t = torch()
    rng = np.random.default_rng(rows + cols)
    g = np.stack([as_type(gradient(rng, rows, cols), to) for _ in range(3)])
    wide = t.full((3, rows + 1, cols + 3), float("nan"), dtype=dtype(to), device="cuda")
    view = wide[:, 1:, 2:-1]
    view.copy_(dev(g.reshape(-1, cols), to).view(3, rows, cols))
    given = view.clone()
    iodf.orthogonalise(view, out=view)
    assert wide.isnan().sum() == wide.numel() - view.numel()
    for x, y in zip(g, view):
        check_orth(y, x, to)
    w = [t.zeros((rows, cols), device="cuda", dtype=dtype(to)) for _ in range(3)]
    m = [t.zeros((rows, cols), device="cuda") for _ in range(3)]
    iodf.muon_step(w, list(given), m, 1.0, beta=0.0, nesterov=False, scale=-1.0)
    for k in range(3):
        assert t.equal(m[k], given[k].float()) and t.equal(w[k], view[k])


@pytest.mark.parametrize("rows,cols", [(128, 128), (70, 100)])
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("grad", NAMES)
def test_muon_step_one_block(rows, cols, name, grad):
    rng = np.random.default_rng(19)
    w, g, m = as_type(rng.standard_normal((rows, cols)) / np.sqrt(cols), name), as_type(gradient(rng, rows, cols), grad), as_type(gradient(rng, rows, cols), "f32")
    wt, mt = dev(w, name), dev(m)
    iodf.muon_step(wt, dev(g, grad), mt, 0.05, beta=0.9, decay=0.2, scale=0.7)
    new = np.float64(np.float32(0.9)) * m + g
    near(mt, new, "f32", 2 * U * (np.abs(m) + np.abs(g)), "momentum")
    step, off = ref.orthogonalise(g + 0.9 * new, parts=name != "bf16")
    want = (1 - 0.05 * 0.2) * w - 0.05 * 0.7 * step
    assert np.linalg.norm(host(wt) - want) <= np.linalg.norm(half_unit(name, want)) + 0.05 * 0.7 * off + 4 * U * np.linalg.norm(w)


@pytest.mark.parametrize("rows", [1, 2, 3, 5, 9, 16, 17])
@pytest.mark.parametrize("classes,cols", [(1, 3), (77, 259), (4100, 1030)])
def test_class_loss_gradients_of_few_rows(rows, classes, cols):
    """In 32 bits a table is read as it lies: strided, any element, padded rows of anything, one gradient or both."""
    t = torch()
    u, w, target, live, rng = some(rows, classes, cols, "f32", seed=23, dead=0.3)
    up = upstream(rng, rows, "both")
    du, dw = check_backward(u, w, target, live, "f32", *up)
    assert t.equal(check_backward(u, w, target, live, "f32", *up, need=(True, False))[0], du)
    assert t.equal(check_backward(u, w, target, live, "f32", *up, need=(False, True))[1], dw)
    wide = t.full((classes, cols + 3), float("nan"), device="cuda")
    wide[:, 1:cols + 1] = dev(w)
    lse = dev(ref.loss(u, w, target, live)[1].astype(np.float32))
    su, st = spoiled(u, target, live)
    again = iodf.class_loss_backward(dev(su), wide[:, 1:cols + 1], long(st), lse, dev(up[0]), dev(up[1]), live=on_gpu(live))
    assert t.equal(again[0], du) and t.equal(again[1], dw)


def test_class_loss_gradients_of_few_rows_and_no_class():
    t = torch()
    u, w, target, _, rng = some(5, 90, 33, "f32", seed=29)
    lse = dev(ref.loss(u, w, target, None)[1].astype(np.float32))
    target[2], target[4] = 90, -1
    du, dw = iodf.class_loss_backward(dev(u), dev(w), long(target), lse, t.ones(5, device="cuda"))
    assert du[[2, 4]].isnan().all() and du[[0, 1, 3]].isfinite().all() and dw.isnan().all()
