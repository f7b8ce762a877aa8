"""Every kernel that the loss over a table of classes and orthogonalising can take (step_plans.py; test_step_plans_cpu.py says that none is left out),
against 64 bits on the card."""
import numpy as np
import pytest

import paper_2206_08869_amd as iodf
import step_plans as plans
import step_ref as ref
from test_gpu_blocks import as_type, dev, dtype, torch
from test_gpu_step import check_orth, gradient, on_card
from test_gpu_step_parts import FINE, few_make_it_up, on_card_gradients

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.mark.parametrize("count,rows,cols,name", plans.ORTH_SHAPES)
def test_orthogonalise_by_every_kernel(count, rows, cols, name):
    """Small ones against the steps with their roundings put in. Of large ones what roundings of h beside the diagonal come to was taken from a simulation of them in 64 bits:
    2 to 3 h; with all numbers in two parts what 32-bit sums come to, 4e-6."""
    t = torch()
    if rows * cols < 1 << 18:
        g = as_type(gradient(np.random.default_rng(rows * 11 + cols), rows, cols), "f32")
        check_orth(iodf.orthogonalise(dev(g), dtype=dtype(name)), g, name)
        return
    gen = t.Generator("cuda").manual_seed(61)
    g = t.randn((count, rows, cols), generator=gen, device="cuda") * t.exp(0.4 * t.randn((cols,), generator=gen, device="cuda"))
    r = iodf.orthogonalise(g, dtype=dtype(name))
    w, m = [t.zeros((rows, cols), dtype=dtype(name), device="cuda") for _ in range(count)], [t.zeros((rows, cols), device="cuda") for _ in range(count)]
    iodf.muon_step(w, list(g), m, 1.0, beta=0.0, nesterov=False, scale=-1.0)
    for k in range(count):
        assert t.equal(w[k], r[k]) and t.equal(m[k], g[k])
    for k in {0, count - 1}:
        x = g[k].double() / g[k].double().norm()
        x = x.t().contiguous() if rows > cols else x
        for _ in range(5):
            p = x @ x.t().contiguous()
            x = 3.4445 * x + (-4.7750 * p + 2.0315 * p @ p) @ x
        x = x.t() if rows > cols else x
        most = {"bf16": 2.0 ** -9 + 4 * 2.0 ** -12, "f16": 2.0 ** -12 + 4e-6, "f32": 4e-6}[name]
        assert (r[k].double() - x).norm() <= most * x.norm() + (2.0 ** -25 * x.numel() ** 0.5 if name == "f16" else 0.0)


def laid(x, aligned):
    """x in rows that start at multiples of 16 bytes, or at any element."""
    t = torch()
    rows, cols = x.shape
    pitch = (cols + 7) // 8 * 8 if aligned else cols + 1
    there = t.full((rows * pitch + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = there[0 if aligned else 1:].as_strided((rows, cols), (pitch, 1))
    view.copy_(x)
    return view


@pytest.mark.parametrize("rows,classes,cols,name,backward,padded,aligned", plans.LOSS_CALLS)
def test_class_loss_by_every_kernel(rows, classes, cols, name, backward, padded, aligned):
    t = torch()
    u, w, target, d = on_card(rows, classes, cols, name, 62)
    live = t.ones(rows, dtype=t.bool, device="cuda")
    if padded:
        live = t.arange(rows, device="cuda") % 5 != 4
        live[0] = rows == 1
    w64, lse, loss, slack = w.double(), [], [], []
    for at in range(0, rows, 16384):
        x = u[at:at + 16384].double()
        s = x @ w64.t().contiguous()
        lse.append(t.logsumexp(s, 1))
        loss.append(lse[-1] - s.gather(1, target[at:at + 16384, None])[:, 0])
        slack.append(64 * U * (x.abs() @ w64.abs().t().contiguous()).amax(1) + 64 * U * (1 + lse[-1].abs() + s.abs().amax(1)))
    lse, loss, slack = (t.cat(v).masked_fill(~live, 0.0) for v in (lse, loss, slack))
    lse32 = lse.float()
    z = d.flip(0).contiguous()
    step = FINE[name] if few_make_it_up(rows, classes, cols, name) else ref.HALF[name]
    least = 2.0 ** -38 * float((d.abs() + z.abs()).max()) if name == "f16" else 0.0
    want = on_card_gradients(u, w, target, lse32, d, z, live, step, least) if backward else None
    if padded:
        u = u.masked_fill(~live[:, None], float("nan"))
        target = target.masked_fill(~live, -(1 << 40))
        d, z, lse32 = (x.masked_fill(~live, float("nan")) for x in (d, z, lse32))
    u, w, mask = laid(u, aligned), laid(w, aligned), live if padded else None
    r = iodf.class_loss(u, w, target, live=mask)
    assert (r.lse.double() - lse).abs().sub(slack).max() <= 0 and (r.loss.double() - loss).abs().sub(2 * slack).max() <= 0
    if not backward:
        return
    got = iodf.class_loss_backward(u, w, target, lse32, d, z, live=mask)
    small = 2.0 ** -25 if name == "f16" else 0.0
    for a, b, off in zip(got, want[:2], want[2:]):
        # what is rounded at the end is at most |b| + off
        assert a.isfinite().all() and ((a.double() - b).abs() - off - HALF[name] * (b.abs() + off) - small).max() <= 0
        # sums of terms of either sign are smaller than their terms' magnitudes: in the norm independent roundings of g and of the result are within half a step each
        assert (a.double() - b).norm() <= max(HALF[name], 2e-6 if name == "f32" else 0.0) * b.norm() + small * b.numel() ** 0.5
    if padded:
        assert not got[0][~live].any()
