"""The differentiable calls as autograd sees them: what they keep, how long, what they notice, and with padded rows."""
import pytest

import paper_2206_08869_amd as iodf

pytestmark = pytest.mark.gpu


def torch():
    import torch as t
    return t


class Block:
    """A stream of `rows` rows through two joins with a gated block between them, as an example of all three calls."""

    def __init__(self, rows=512, cols=96, hid=160, live=None):
        t = torch()
        gen = t.Generator("cuda").manual_seed(rows)

        def leaf(*shape, by=1.0, plus=0.0):
            return (by * t.randn(shape, generator=gen, device="cuda") + plus).requires_grad_()

        self.h, self.f = leaf(rows, cols), leaf(rows, cols)
        self.w1, self.w2 = leaf(2 * hid, cols, by=0.1), leaf(cols, hid, by=0.1)
        self.joins = [[leaf(1, plus=0.5, by=0.0), leaf(cols, by=0.1, plus=0.7), leaf(cols, by=0.1, plus=1.0), leaf(cols, by=0.1, plus=1.0)]
                      for _ in range(2)]
        self.dy = t.randn((rows, cols), generator=gen, device="cuda")
        self.live, self.rows = live, None if live is None else live.clone()  # the loss has a mask of its own

    def leaves(self):
        return [self.h, self.f, self.w1, self.w2, *self.joins[0], *self.joins[1]]

    def loss(self, seen=None):
        first, second = self.joins
        h, u, codes = iodf.joined(self.h, self.f, *first, live=self.live)
        ab = iodf.projection(u, self.w1, codes, col_scale=first[3].detach(), live=self.live)
        f = iodf.gated_projection(ab, self.w2, live=self.live)
        h, u, last = iodf.joined(h, f, *second, live=self.live)
        if seen is not None:
            seen += [codes, last]
        out = (h + u) * self.dy
        return (out if self.rows is None else out[self.rows]).sum()


def test_the_backward_pass_lets_checkpoints_go():
    """While the loss, and with it the graph, is still held, as in a training loop until the next step's loss takes its place."""
    t = torch()
    rows, cols, hid = 8192, 512, 1024
    block = Block(rows, cols, hid)
    t.autograd.grad(block.loss(), block.leaves())  # what the libraries allocate once
    t.cuda.synchronize()
    before = t.cuda.memory_allocated()
    loss = block.loss()
    kept = t.cuda.memory_allocated() - before
    codes = rows * (4 * cols + 2 * hid) * 33 // 32  # of two joins and of a gated activation
    assert kept >= codes
    loss.backward()
    for x in block.leaves():
        x.grad = None
    t.cuda.synchronize()
    assert t.cuda.memory_allocated() - before < codes // 16 and loss.requires_grad


def test_saved_tensor_hooks_see_the_checkpoints():
    """Offloading and the like work on saved tensors: every checkpoint passes through them, and what they give back is used."""
    t = torch()
    block = Block()
    want = t.autograd.grad(block.loss(), block.leaves())
    packed = []

    def pack(x):
        packed.append(x.dtype)
        return x.cpu()

    with t.autograd.graph.saved_tensors_hooks(pack, lambda x: x.cuda()):
        loss = block.loss()
    got = t.autograd.grad(loss, block.leaves())
    assert packed.count(t.int8) == 7  # x and n of two joins, x for the projection, a and b
    for a, b in zip(got, want):
        assert t.equal(a, b)


@pytest.mark.parametrize("what", ["live", "codes.q", "codes.e"])
def test_what_is_changed_in_place_between_the_passes_is_an_error(what):
    t = torch()
    live = t.rand(512, device="cuda") < 0.8
    block, seen = Block(live=live), []
    loss = block.loss(seen)
    if what == "live":
        live.fill_(True)
    else:
        getattr(seen[0], what[-1]).add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_a_projection_whose_weight_learns_wants_codes():
    t = torch()
    u, w = t.randn((4, 32), device="cuda"), t.randn((8, 32), device="cuda").requires_grad_()
    with pytest.raises(ValueError):
        iodf.projection(u, w, None)
    assert t.equal(iodf.projection(u, w.detach(), None), u @ w.detach().t())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_padded_rows_through_the_differentiable_calls(dtype):
    """Gradients of a batch with padded rows are those of the batch without them, whatever stands in the padded rows; as near as sums over
    other rows in another order and other kernels of the projections' library come to each other."""
    t = torch()
    rows = 640
    live = t.rand(rows, generator=t.Generator("cuda").manual_seed(1), device="cuda") < 0.7
    block = Block(rows, live=live)
    whole = Block(rows)
    for x in (block, whole):
        x.h, x.f = (v.detach().to(getattr(t, dtype)) for v in (x.h, x.f))
    whole.h, whole.f, whole.dy = whole.h[live], whole.f[live], whole.dy[live]
    block.f[~live] = float("nan")
    block.h[~live] = float("inf")
    for x in (block, whole):
        x.h.requires_grad_(), x.f.requires_grad_()
    got = t.autograd.grad(block.loss(), block.leaves())
    want = t.autograd.grad(whole.loss(), whole.leaves())
    for k, (g, w) in enumerate(zip(got, want)):
        if k < 2:
            assert not g[~live].any()
            g = g[live]
        assert t.isfinite(g).all()
        # activations in 32 bits: a code on a border may fall to either side; in 16: other products' roundings besides
        assert (g - w).float().norm() <= (0.02 if dtype == "bfloat16" else 0.01) * w.float().norm()


def test_outputs_that_are_given_are_known_to_have_changed():
    """A tensor that autograd keeps for another operation, overwritten as h_out or out, is an error in that one's backward pass."""
    t = torch()
    h, f, w = (t.randn(s, device="cuda") for s in ((8, 32), (8, 32), (24, 32)))
    other, codes, dy = t.randn((8, 32), device="cuda").requires_grad_(), iodf.pack(f), t.randn((8, 24), device="cuda")
    for overwrite, kept in ((lambda: iodf.join(h, f, save=False, h_out=h), h), (lambda: iodf.join(f, f, h_out=h[:, :]), h),
                            (lambda: iodf.weight_grad(codes, dy, out=w, accumulate=True), w)):
        loss = (other * kept[:8]).sum()
        overwrite()
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
    with t.inference_mode():
        x = t.ones((3, 32), device="cuda")
        assert iodf.join(x, x, save=False, h_out=x)[0] is x and (x == 2).all()


def test_calls_that_record_no_graph_refuse_what_would_need_one():
    """Activations and gradients that require a gradient, while autograd records. Parameters may require one; whole numbers have none."""
    t = torch()
    x, g = t.randn((8, 32), device="cuda"), t.randn((8, 32), device="cuda").requires_grad_()
    w = t.ones(32, device="cuda").requires_grad_()
    codes = iodf.pack(x)
    _, _, saved = iodf.join(x, x, w_pre=w)
    _, gated = iodf.glu(x, x)
    calls = (lambda: iodf.join(g, x), lambda: iodf.join(x, g), lambda: iodf.join(x, x, h_out=g), lambda: iodf.join_backward(saved, g, x, w_pre=w),
             lambda: iodf.join_backward(saved, x, g, w_pre=w), lambda: iodf.glu(g, x), lambda: iodf.glu(x, g),
             lambda: iodf.glu_backward(gated, g), lambda: iodf.weight_grad(codes, g), lambda: iodf.weight_grad(codes, x, out=t.zeros_like(g).expand(
                 8, 32).repeat(4, 1).requires_grad_()))
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with t.no_grad():
            call()
    iodf.join_backward(saved, x, x, w_pre=w), iodf.weight_grad(codes, x, col_scale=w), iodf.pack(g)


def test_gradients_that_nobody_asked_for_are_not_computed(monkeypatch):
    """A projection of data, and a frozen weight; nothing is kept where nothing is recorded."""
    t = torch()
    from paper_2206_08869_amd import blocks
    rows, cols, out = 4096, 1024, 16
    x, dy = t.randn((rows, cols), device="cuda"), t.randn((rows, out), device="cuda")
    w = t.randn((out, cols), device="cuda")
    codes = iodf.pack(x)
    learning, data = w.clone().requires_grad_(), x.clone().requires_grad_()
    y = iodf.projection(x, learning, codes)
    want = iodf.weight_grad(codes, dy)
    t.cuda.synchronize()
    t.cuda.reset_peak_memory_stats()
    before = t.cuda.memory_allocated()
    got, = t.autograd.grad(y, learning, dy)
    assert t.equal(got, want) and t.cuda.max_memory_allocated() - before < 4 * rows * cols  # no gradient of x

    def never(*args, **more):
        raise AssertionError("a weight gradient that nobody asked for")

    a = t.randn((rows, 2 * out), device="cuda").requires_grad_()
    frozen = t.randn((cols, out), device="cuda")
    both = t.autograd.grad(iodf.gated_projection(a, frozen.clone().requires_grad_()), a, x)[0]
    monkeypatch.setattr(blocks, "weight_grad", never)
    assert t.equal(t.autograd.grad(iodf.projection(data, w, codes), data, dy)[0], dy @ w)
    assert t.equal(t.autograd.grad(iodf.gated_projection(a, frozen), a, x)[0], both)
    saves, glu = [], blocks.glu
    monkeypatch.setattr(blocks, "glu", lambda *args, save=True, **more: saves.append(save) or glu(*args, save=save, **more))
    with t.no_grad():
        silent = iodf.gated_projection(a, frozen)
    assert t.equal(silent, iodf.gated_projection(a, frozen).detach()) and not silent.requires_grad
    assert t.equal(silent, iodf.gated_projection(a.detach(), frozen)) and saves == [False, True, False]


@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("inputs", ["float32", "bfloat16"])
def test_projections_under_autocast(kind, inputs):
    """The product's type is autocast's, the gradients' are the inputs'; near the product of the same numbers in 64 bits: 16-bit roundings of the
    operands (half a unit, 2^-9, each), of the product and of its gradient, and codes of a percent or so."""
    t = torch()
    gen = t.Generator("cuda").manual_seed(1)
    x, a = (t.randn((256, 96), generator=gen, device="cuda").to(getattr(t, inputs)).requires_grad_() for _ in range(2))
    w, v = t.randn((64, 96), generator=gen, device="cuda").requires_grad_(), t.randn((64, 48), generator=gen, device="cuda").requires_grad_()
    dy = t.randn((256, 64), generator=gen, device="cuda").to(getattr(t, kind))
    with t.autocast("cuda", dtype=getattr(t, kind)):
        y, z = iodf.projection(x, w, iodf.pack(x)), iodf.gated_projection(a, v)
    assert y.dtype == z.dtype == getattr(t, kind)
    got = t.autograd.grad((y, z), (x, w, a, v), (dy, dy))
    wide = [p.detach().double().requires_grad_() for p in (x, w, a, v)]
    x2, w2, a2, v2 = wide
    left, right = a2.chunk(2, 1)
    want = t.autograd.grad((x2 @ w2.t(), (left * t.sigmoid(left) * right) @ v2.t()), wide, (dy.double(), dy.double()))
    for g, w, p in zip(got, want, (x, w, a, v)):
        assert g.dtype == p.dtype and (g.double() - w).norm() <= 0.03 * w.norm()


def test_a_projection_that_nothing_is_recorded_of_wants_no_codes():
    t = torch()
    u, w = t.randn((4, 32), device="cuda").requires_grad_(), t.randn((8, 32), device="cuda").requires_grad_()
    with t.no_grad():
        y = iodf.projection(u, w, None)
    assert t.equal(y, (u @ w.t()).detach()) and not y.requires_grad
    got, = t.autograd.grad(iodf.projection(u, w.detach(), None), u, t.ones_like(y))
    assert t.equal(got, t.ones_like(y) @ w.detach())
