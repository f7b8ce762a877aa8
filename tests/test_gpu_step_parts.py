"""Gradients of the loss over a table of classes by the way they are computed: g in one part, in two and in three, one piece of the classes and several, whole
tiles and slices. Against formulas in 64 bits, element by element; bounds come from how many bits g has (step_ref.py)."""
import numpy as np
import pytest

import paper_2206_08869_amd as iodf
import step_ref as ref
from test_gpu_blocks import dev, dtype, half_unit, host, near, on_gpu, torch
from test_gpu_step import NAMES, SHAPES, long, on_card, some, spoiled, upstream

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# Of g where few numbers of it make up a gradient: half a step of two parts in 16 bits, of the sums in 32.
FINE = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22, "f32": 2.0 ** -24}


def few_make_it_up(rows, classes, cols, name):
    """Where iodf.h says that g has two parts (in 32 bits it always has all)."""
    return name == "f32" or rows <= 16 or classes <= 32 or cols <= 128 or rows * classes <= 65536


def rounded(want, slack, name):
    """slack, and what the result's rounding may be more than half a step at `want`. The number that is rounded is up to slack away from want, so at most |want| + slack, and
    steps grow with numbers: want = 2^-10.0005 and slack 4.8e-6 in bfloat16 may be 0.00098038, past 2^-10, where half a step is 3.8e-6 and not 1.9e-6."""
    return slack + 1.01 * (half_unit(name, np.abs(want) + slack) - half_unit(name, want))


def check(u, w, target, live, name, up):
    lse = ref.loss(u, w, target, live)[1].astype(np.float32)
    su, st = spoiled(u, target, live)
    on = lambda a: None if a is None else dev(np.where(live, a, np.nan) if live is not None else a)  # noqa: E731
    got = iodf.class_loss_backward(dev(su, name), dev(w, name), long(st), on(lse), on(up[0]), on(up[1]), live=on_gpu(live))
    du, dw, eu, ew = ref.loss_backward(u, w, target, lse.astype(np.float64), *up, live, name)
    near(got[0], du, name, rounded(du, eu, name), "du")
    near(got[1], dw, name, rounded(dw, ew, name), "dweight")
    return got


ONE_PART = [(300, 513, 200), (1000, 700, 264), (17, 4001, 1030), (2000, 33, 129), (257, 256, 520)]


@pytest.mark.parametrize("rows,classes,cols", ONE_PART)
@pytest.mark.parametrize("dead", [None, 0.3])
@pytest.mark.parametrize("kind", ["both", "loss", "lse"])
@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_gradients_of_one_part(rows, classes, cols, name, dead, kind):
    assert not few_make_it_up(rows, classes, cols, name)
    u, w, target, live, rng = some(rows, classes, cols, name, seed=51, dead=dead)
    check(u, w, target, live, name, upstream(rng, rows, kind))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("rows,classes,cols", [(300, 513, 200), (500, 300, 256)])
def test_gradients_of_one_part_strided_at_any_element(rows, classes, cols, name):
    """Rows with gaps that start at any element give the bits of rows of their own; what lies between them is not read, and gradients are rows of their own."""
    t = torch()
    u, w, target, live, rng = some(rows, classes, cols, name, seed=52, dead=0.2)
    su, st = spoiled(u, target, live)
    up = upstream(rng, rows, "both")
    base = check(u, w, target, live, name, up)
    lse = dev(ref.loss(u, w, target, live)[1].astype(np.float32))
    for gap, first in ((0, 1), (3, 0), (8, 8), (5, 3)):
        us = t.full((rows * (cols + gap) + 16,), float("nan"), dtype=dtype(name), device="cuda")
        ws = t.full((classes * (cols + gap) + 16,), float("nan"), dtype=dtype(name), device="cuda")
        uv, wv = us[first:].as_strided((rows, cols), (cols + gap, 1)), ws[first:].as_strided((classes, cols), (cols + gap, 1))
        uv.copy_(dev(su, name)), wv.copy_(dev(w, name))
        got = iodf.class_loss_backward(uv, wv, long(st), lse, dev(up[0]), dev(up[1]), live=on_gpu(live))
        assert t.equal(got[0], base[0]) and t.equal(got[1], base[1])


@pytest.mark.parametrize("name", NAMES)
def test_gradients_of_one_part_and_targets_that_are_no_class(name):
    u, w, target, live, rng = some(300, 513, 200, name, seed=53, dead=0.2)
    live[[3, 270]] = True
    lse = dev(ref.loss(u, w, target, live)[1].astype(np.float32))
    su, st = spoiled(u, target, live)
    st[3], st[270] = 513, -1
    du, dw = iodf.class_loss_backward(dev(su, name), dev(w, name), long(st), lse, dev(np.full(300, 0.01)), live=on_gpu(live))
    rest = np.ones(300, bool)
    rest[[3, 270]] = False
    assert np.isnan(host(du)[~rest]).all() and np.isfinite(host(du)[rest]).all() and not host(du)[~live].any() and np.isnan(host(dw)).all()


@pytest.mark.parametrize("rows,classes,cols", SHAPES + [(21, 600, 300), (40, 1600, 700)])
@pytest.mark.parametrize("name", NAMES)
def test_gradients_that_few_numbers_make_up_have_all_their_bits(rows, classes, cols, name):
    """A result may be off by its own rounding and by next to nothing of g's: the bound is broken where a second part of g is lost (test_step_parts_cpu.py)."""
    if not few_make_it_up(rows, classes, cols, name):
        pytest.skip("g has one part")
    u, w, target, live, rng = some(rows, classes, cols, name, seed=54)
    up = upstream(rng, rows, "both")
    lse = ref.loss(u, w, target, live)[1].astype(np.float32)
    got = iodf.class_loss_backward(dev(u, name), dev(w, name), long(target), dev(lse), dev(up[0]), dev(up[1]))
    least = 2.0 ** -38 * max(np.abs(up[0]).max(), np.abs(up[0] + up[1]).max()) if name == "f16" else 0.0
    du, dw, eu, ew = ref.gradients_by_the_parts(u, w, target, lse.astype(np.float64), *up, live, FINE[name], least)
    near(got[0], du, name, rounded(du, eu, name), "du")
    near(got[1], dw, name, rounded(dw, ew, name), "dweight")


def on_card_gradients(u, w, target, lse, d, z, live, step, least):
    """step_ref.gradients_by_the_parts on the card, some rows at a time: du, dw, and what each may be off by."""
    t = torch()
    w64, parts = w.double(), []
    dw, ew = t.zeros(w.shape, dtype=t.float64, device="cuda"), t.zeros(w.shape, dtype=t.float64, device="cuda")
    for at in range(0, len(u), 16384):
        here = slice(at, at + 16384)
        there = live[here]
        x = u[here].double().masked_fill(~there[:, None], 0.0)
        up, both = d[here].double() * there, (d[here].double() + z[here].double()) * there
        s = x @ w64.t().contiguous()
        p = t.exp(s - lse[here].double()[:, None]).masked_fill(~there[:, None], 0.0) * both[:, None]
        g = p.clone()
        g.scatter_add_(1, target[here].clamp(0, len(w) - 1)[:, None], -up[:, None])
        off = p.abs() * (64 * U * (x.abs() @ w64.abs().t().contiguous()) + 16 * U * (1 + s.abs())) + g.abs() * (step + 64 * U) + least * there[:, None]
        parts.append((g @ w64, off @ w64.abs()))
        dw += g.t().contiguous() @ x
        ew += off.t().contiguous() @ x.abs()
    return t.cat([p[0] for p in parts]), dw, t.cat([p[1] for p in parts]), ew


@pytest.mark.parametrize("rows,classes,cols,name", [(131072, 2500, 136, "bf16"), (131072, 2500, 136, "f16"), (131072, 2500, 130, "bf16"), (65536, 3000, 136, "f32"),
                                                   (131072, 2300, 64, "f16")])
@pytest.mark.parametrize("padded", [False, True])
def test_gradients_of_several_pieces(rows, classes, cols, name, padded):
    """g of all classes does not fit 512 MB: pieces, the last one shorter, with targets and a penalty's gradients in every one."""
    t = torch()
    u, w, target, d = on_card(rows, classes, cols, name, 55)
    z = d.flip(0).contiguous()
    lse = iodf.class_loss(u, w, target).lse
    live = t.ones(rows, dtype=t.bool, device="cuda")
    if padded:
        live = t.arange(rows, device="cuda") % 7 != 3
    step = FINE[name] if few_make_it_up(rows, classes, cols, name) else ref.HALF[name]
    least = 2.0 ** -38 * float((d.abs() + z.abs()).max()) if name == "f16" else 0.0
    want = on_card_gradients(u, w, target, lse, d, z, live, step, least)
    if padded:
        u[~live] = float("nan")
        target = target.masked_fill(~live, -(1 << 40))
        lse, d, z = (x.masked_fill(~live, float("nan")) for x in (lse, d, z))
    got = iodf.class_loss_backward(u, w, target, lse, d, z, live=live if padded else None)
    half = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[name]
    small = 2.0 ** -25 if name == "f16" else 0.0
    for a, b, off in zip(got, want[:2], want[2:]):
        assert a.isfinite().all() and ((a.double() - b).abs() - off - half * b.abs() - small).max() <= 0
        # sums of terms of either sign are smaller than their terms' magnitudes: in the norm independent roundings of g and of the result are within half a step each
        assert (a.double() - b).norm() <= max(half, 2e-6 if name == "f32" else 0.0) * b.norm() + small * b.numel() ** 0.5
    if padded:
        assert not got[0][~live].any()
