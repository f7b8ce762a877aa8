"""Padded rows and no rows at all, in the training operators: whatever stands in a padded row's operands stays out of every result."""
import numpy as np
import pytest

import paper_2206_08869_amd as iodf

pytestmark = pytest.mark.gpu


def torch():
    import torch as t
    return t


def padded_codes(x, live):
    """The codes of x, and the same with padded rows that stand for NaN, infinity (both e = 255) or the largest values there are."""
    t = torch()
    clean = iodf.pack(x, live=live)
    q, e = clean.q.clone(), clean.e.clone()
    dead = ~live
    q[dead] = t.randint(-127, 128, q[dead].shape, device="cuda", dtype=t.int8)
    e[dead] = t.where(t.rand(e[dead].shape, device="cuda") < 0.5, 255, 254).to(t.uint8)
    return clean, iodf.Codes(q, e, x.shape[1])


# every tile: narrow and wide sides, layers of 256 x 256 tiles with whole and ragged slices, rows on both sides of a tile's end
@pytest.mark.parametrize("rows,cols,out,name", [
    (1, 32, 8, "float32"), (31, 33, 65, "bfloat16"), (1000, 72, 130, "bfloat16"), (700, 40, 24, "float16"), (5000, 200, 40, "float32"),
    (4099, 512, 264, "bfloat16"), (3000, 1030, 1100, "float32"), (4100, 300, 1030, "float16"), (70000, 16, 16, "bfloat16"),
    (1025, 2048, 2048, "bfloat16"), (9001, 2050, 2100, "bfloat16"), (16384, 2048, 2048, "bfloat16"), (131073, 264, 392, "bfloat16")])
def test_weight_grad_leaves_a_padded_row_s_codes_out(rows, cols, out, name):
    t = torch()
    gen = t.Generator("cuda").manual_seed(rows + cols)
    live = t.rand(rows, generator=gen, device="cuda") < 0.7
    live[-1] = False
    x = t.randn((rows, cols), generator=gen, device="cuda")
    dy = t.randn((rows, out), generator=gen, device="cuda").to(getattr(t, name))
    dy[~live] = float("nan")
    clean, dirty = padded_codes(x, live)
    want = iodf.weight_grad(clean, dy, live=live)
    got = iodf.weight_grad(dirty, dy, live=live)
    assert t.isfinite(want).all() and t.equal(got, want)


def test_projection_leaves_padded_rows_out_of_its_weight_s_gradient():
    """A checkpoint that was packed without the mask, of a tensor whose padded rows hold NaN and infinities."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(2)
    x, dy = (t.randn((300, n), generator=gen, device="cuda").bfloat16() for n in (72, 40))
    w = t.randn((40, 72), generator=gen, device="cuda").requires_grad_()
    live = t.rand(300, generator=gen, device="cuda") < 0.6
    want = iodf.weight_grad(iodf.pack(x, live=live), dy, live=live)
    x[~live] = float("nan")
    x[~live, 40:] = float("inf")
    got, = t.autograd.grad(iodf.projection(x, w, iodf.pack(x), live=live), w, dy)
    assert np.isfinite(want.cpu().numpy()).all() and t.equal(got, want)


@pytest.mark.parametrize("groups", [1, 3, 200])
@pytest.mark.parametrize("cols", [5, 72, 9000])
def test_join_backward_of_no_rows_gives_zeros(groups, cols):
    """For every gate there is, in memory that held other numbers just before."""
    t = torch()
    h = t.empty((0, cols), device="cuda")
    par = [t.ones(s, device="cuda") for s in ((1,), (groups, cols), (cols,), (cols,))]
    _, u, saved = iodf.join(h, h, *par)
    junk = [t.full((groups, cols), float("nan"), device="cuda") for _ in range(8)]
    del junk
    g = iodf.join_backward(saved, h, u, *par)
    for got, p in zip(g[2:], par):
        assert t.equal(got, t.zeros_like(p))


@pytest.mark.parametrize("rows,cols", [(1, 40), (50, 40), (33, 300), (20, 1111), (9, 9001)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_join_leaves_a_padded_row_s_gate_out(rows, cols, kind):
    """A gate for each row, no number where the row is padding: h' is h there to the bit (signs of zeros among them), nothing reaches a gradient."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(rows)
    live = t.rand(rows, generator=gen, device="cuda") < 0.6
    live[0] = rows > 1
    h, f, dh, du = (t.randn((rows, cols), generator=gen, device="cuda").to(getattr(t, kind)) for _ in range(4))
    h[:, ::3] = -0.0
    clean = [t.randn(s, generator=gen, device="cuda") for s in ((1,), (rows, cols), (cols,), (cols,))]
    dirty = [x.clone() for x in clean]
    dirty[1][~live] = float("nan")
    dirty[1][~live, ::2] = float("inf")
    bits = t.int32 if kind == "float32" else t.int16

    def same(a, b):
        return t.equal(a.view(bits), b.view(bits)) if a.dtype == h.dtype else t.equal(a, b)

    (h1, u1, s1), (h2, u2, s2) = (iodf.join(h, f, *par, live=live) for par in (clean, dirty))
    assert same(h1, h2) and same(u1, u2) and same(h1[~live], h[~live]) and not u1[~live].any()
    for a, b in zip((*s1.x[:2], *s1.n[:2], s1.inv_pre, s1.inv_post), (*s2.x[:2], *s2.n[:2], s2.inv_pre, s2.inv_post)):
        assert t.equal(a, b)
    g1, g2 = (iodf.join_backward(s1, dh, du, *par, live=live) for par in (clean, dirty))
    for a, b in zip(g1, g2):
        assert t.isfinite(a).all() and same(a, b)
